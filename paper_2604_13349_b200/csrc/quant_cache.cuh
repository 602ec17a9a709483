// A relayed cache held in 8 or 4 bits: the cache as the kernels see it, writing rows to it and reading rows back.
//
// 8 bits: x = code * scale with scale = max |x| / 127 over the row (the format of the int8 copy that the compression makes).
// 4 bits: the channels of a row fall into D / 32 groups of 32, group(c) = (c / 4) mod (D / 32), with a scale each,
// max |x| / 7 rounded to five significant bits.  Five bits times a code of three: a value is a bf16 number, so that whoever reads
// rows back in bf16 holds what the attention on codes sees.  And five bits tell codes apart for good: 2 x and an odd multiple of
// such a scale, if they differ, differ by at least 2^-24 of either, so the fp32 quotient x / scale lies on the same side of
// n + 1/2 as the real one, and the codes are those of exact arithmetic.
// The groups are taken across the row so that the eight lanes that share a channel tile of the attention's second product
// hold channels of every group while a row's codes stay in order.
#pragma once

#include "attend_common.cuh"

namespace obf {

struct QuantDev {
    const uint8_t *k, *v;                  // codes
    const uint8_t *k_scale, *v_scale;
    long long ks[3], vs[3], kss[3], vss[3];   // bytes from one sequence, head and row to the next
};

template <int BITS, int D>
struct QuantRow {
    static constexpr int BYTES = D * BITS / 8;
    static constexpr int GROUPS = BITS == 4 ? D / 32 : 1;
    static constexpr int SCALE_BYTES = BITS == 4 ? 2 * GROUPS : 4;
};

// Whole-number division of numbers below 2^31 by one that the host knows: x / d = hi32(x * mul) >> shift with
// mul = ceil(2^(32 + shift) / d), 2^shift < d <= 2^(shift + 1) (d > 1), whose error stays below 1 / d for such x.
struct FastDiv {
    uint32_t d, mul;
    int32_t shift;
};

inline FastDiv fast_div(uint32_t d)
{
    FastDiv f = {d, 0u, 0};
    if (d < 2) return f;
    while ((2ull << f.shift) < d) ++f.shift;
    f.mul = (uint32_t)(((1ull << (32 + f.shift)) + d - 1) / d);
    return f;
}

__device__ __forceinline__ uint32_t div_by(uint32_t x, const FastDiv &f) { return f.mul ? __umulhi(x, f.mul) >> f.shift : x; }

// Rows of a call, K's first, then V's: (sequence, head) after (sequence, head), row after row.
struct RowsDev {
    const void *k, *v;                     // rows to write, or
    void *k_out, *v_out;                   // rows read back / the values of the rows written, or null
    long long ks[3], vs[3], kos[3], vos[3];   // elements
    const int32_t *lens, *new_lens;
    int32_t rows, first, capacity;
    uint32_t total, half;                  // rows of K and V, of one of them
    FastDiv by_rows, by_heads;
};

constexpr int QC_NT = 256;
constexpr int QC_AHEAD = 4;                // rows of a thread in flight

// x * 1 / scale rounded to a whole number as the quotient would be.  bf16 numbers over a scale of five bits: the quotient is n + 1/2
// exactly or at least 1/496 away from it (2 x and (2 n + 1) scale are multiples of an eighth of the scale's last bit), so rounding the
// product to a multiple of 2^-10 first undoes its error of 2^-21.  fp32 numbers are divided.
template <typename T>
__device__ __forceinline__ float code4(float x, float scale, float inv)
{
    if constexpr (sizeof(T) == 4) return rintf(__fdiv_rn(x, scale));
    constexpr float GRID = 12288.f;        // 1.5 * 2^13
    return rintf(__fadd_rn(__fadd_rn(x * inv, GRID), -GRID));
}

// 8 bits: the code is the whole number nearest to the fp32 quotient, from which the product is off by at most 2.3e-5.
__device__ __forceinline__ float code8(float x, float scale, float inv)
{
    const float pr = x * inv;
    float v = rintf(pr);
    if (fabsf(fabsf(pr - v) - 0.5f) < 2.44140625e-4f) v = rintf(__fdiv_rn(x, scale));
    return v;
}

// Scale of numbers whose largest magnitude has the bits `top` (as integers, so that what is not a number counts as the largest): not a
// number where one of them is not finite, zero where all are below 2^-110, whose scale would lose bits.
template <int BITS>
__device__ __forceinline__ float scale_of(uint32_t top)
{
    if (top >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    if (top < (127u - 110u) << 23) return 0.f;
    const float x = __uint_as_float(top);
    if constexpr (BITS == 8) return __fdiv_rn(x, 127.f);
    const uint32_t i = __float_as_uint(__fdiv_rn(x, 7.f));
    return __uint_as_float((i + 0x3ffffu + ((i >> 19) & 1u)) & 0xfff80000u);
}

template <typename T>
struct Eight {                             // eight neighbouring channels of a row
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        if constexpr (sizeof(T) == 4) {
            const uint32_t u[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(u[i]);
        } else {
            const uint32_t u[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
        }
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[8])
    {
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
        } else {
            *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        }
    }
};

// Where row f of a call stands: in K or V, its sequence and head, its number.
struct RowAt {
    bool of_v;
    uint32_t b, h, i;
};

__device__ __forceinline__ RowAt row_at(const RowsDev &p, uint32_t f)
{
    RowAt r;
    r.of_v = f >= p.half;
    const uint32_t x = r.of_v ? f - p.half : f, bh = div_by(x, p.by_rows);
    r.i = x - bh * p.by_rows.d;
    r.b = div_by(bh, p.by_heads);
    r.h = bh - r.b * p.by_heads.d;
    return r;
}

// Writing: D / 8 lanes a row, eight channels each; a thread's rows are all read before the first of them is worked on.  Bound by HBM where there
// are many rows, by the latency of a launch and two dependent reads where there are few.
template <typename T, int BITS, int D, bool VALUES>
__global__ void __launch_bounds__(QC_NT) k_quant_write(const __grid_constant__ RowsDev p, const __grid_constant__ QuantDev c)
{
    pdl_wait();
    pdl_trigger();
    constexpr int L = D / 8, R = QC_NT / L;              // lanes of a row, rows of a block at a time
    const int l = threadIdx.x % L;
    const uint32_t f0 = blockIdx.x * (R * QC_AHEAD) + threadIdx.x / L;
    Eight<T> in[QC_AHEAD];
    RowAt at[QC_AHEAD];
    int pos[QC_AHEAD];                                    // row of the cache, or -1: not written
#pragma unroll
    for (int u = 0; u < QC_AHEAD; ++u) {
        const uint32_t f = f0 + u * R;
        pos[u] = -1;
        in[u] = {};
        if (f >= p.total) continue;
        at[u] = row_at(p, f);
        const int n_new = p.new_lens ? min(max(p.new_lens[at[u].b], 0), p.rows) : p.rows;
        const long long to = (long long)(p.lens ? p.lens[at[u].b] : n_new) - n_new + at[u].i;
        if ((int)at[u].i >= n_new || to < 0 || to >= p.capacity) continue;
        pos[u] = (int)to;
        const long long *s = at[u].of_v ? p.vs : p.ks;
        in[u].load(static_cast<const T *>(at[u].of_v ? p.v : p.k) + at[u].b * s[0] + at[u].h * s[1] + at[u].i * s[2] + 8 * l);
    }
#pragma unroll
    for (int u = 0; u < QC_AHEAD; ++u) {
        float x[8], y[8];
        in[u].get(x);
        uint32_t top[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) top[i / 4] = max(top[i / 4], __float_as_uint(x[i]) & 0x7fffffffu);
        if constexpr (BITS == 8) top[0] = max(top[0], top[1]);
#pragma unroll
        for (int w = BITS == 4 && D == 128 ? 2 : 1; w < L; w <<= 1) {
            top[0] = max(top[0], __shfl_xor_sync(0xffffffffu, top[0], w));
            if constexpr (BITS == 4) top[1] = max(top[1], __shfl_xor_sync(0xffffffffu, top[1], w));
        }
        if (pos[u] < 0) continue;
        uint8_t *code = const_cast<uint8_t *>(at[u].of_v ? c.v : c.k), *scale = const_cast<uint8_t *>(at[u].of_v ? c.v_scale : c.k_scale);
        const long long *cs = at[u].of_v ? c.vs : c.ks, *ss = at[u].of_v ? c.vss : c.kss;
        code += at[u].b * cs[0] + at[u].h * cs[1] + pos[u] * cs[2];
        scale += at[u].b * ss[0] + at[u].h * ss[1] + pos[u] * ss[2];
        float s[2], inv[2];
#pragma unroll
        for (int g = 0; g < (BITS == 4 ? 2 : 1); ++g) {
            s[g] = scale_of<BITS>(top[g]);
            inv[g] = s[g] > 0.f ? __frcp_rn(s[g]) : 0.f;
        }
        uint32_t word[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int g = BITS == 4 ? i / 4 : 0;
            float v = 0.f;                                // zeros where the scale is zero or not a number
            if (s[g] > 0.f) v = BITS == 4 ? code4<T>(x[i], s[g], inv[g]) : code8(x[i], s[g], inv[g]);
            y[i] = v * s[g];
            if constexpr (BITS == 4) word[0] |= (uint32_t)((int)v + 8) << (4 * i);
            else word[i / 4] |= (uint32_t)((int)v & 255) << (8 * (i % 4));
        }
        if constexpr (BITS == 4) {
            *reinterpret_cast<uint32_t *>(code + 4 * l) = word[0];
            if (l < D / 64) *reinterpret_cast<uint32_t *>(scale + 4 * l) = __float_as_uint(s[0]) >> 16 | (__float_as_uint(s[1]) & 0xffff0000u);
        } else {
            *reinterpret_cast<uint2 *>(code + 8 * l) = make_uint2(word[0], word[1]);
            if (l == 0) *reinterpret_cast<float *>(scale) = s[0];
        }
        if constexpr (VALUES) {
            const long long *s3 = at[u].of_v ? p.vos : p.kos;
            Eight<T>::store(static_cast<T *>(at[u].of_v ? p.v_out : p.k_out) + at[u].b * s3[0] + at[u].h * s3[1] + at[u].i * s3[2] + 8 * l, y);
        }
    }
}

// Eight neighbouring channels' values from their codes (a word, two words) and scales.
template <int BITS>
__device__ __forceinline__ void values8(float (&y)[8], uint2 code, float s0, float s1)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (BITS == 4) y[i] = (float)((int)(code.x >> (4 * i) & 15u) - 8) * (i < 4 ? s0 : s1);
        else y[i] = (float)(int8_t)((i < 4 ? code.x : code.y) >> (8 * (i % 4))) * s0;
    }
}

// Reading rows first .. first + rows - 1 back, laid out as for writing.
template <typename T, int BITS, int D>
__global__ void __launch_bounds__(QC_NT) k_quant_read(const __grid_constant__ RowsDev p, const __grid_constant__ QuantDev c)
{
    pdl_wait();
    pdl_trigger();
    constexpr int L = D / 8, R = QC_NT / L;
    const int l = threadIdx.x % L;
    const uint32_t f0 = blockIdx.x * (R * QC_AHEAD) + threadIdx.x / L;
    uint2 code[QC_AHEAD];
    float s[QC_AHEAD][2];
    RowAt at[QC_AHEAD];
    bool real[QC_AHEAD];
#pragma unroll
    for (int u = 0; u < QC_AHEAD; ++u) {
        const uint32_t f = f0 + u * R;
        real[u] = f < p.total;
        if (!real[u]) continue;
        at[u] = row_at(p, f);
        const int j = p.first + (int)at[u].i, n = p.lens ? min(p.lens[at[u].b], p.capacity) : p.capacity;
        real[u] = j < n;
        if (!real[u]) continue;
        const long long *cs = at[u].of_v ? c.vs : c.ks, *ss = at[u].of_v ? c.vss : c.kss;
        const uint8_t *from = (at[u].of_v ? c.v : c.k) + at[u].b * cs[0] + at[u].h * cs[1] + j * cs[2];
        const uint8_t *scale = (at[u].of_v ? c.v_scale : c.k_scale) + at[u].b * ss[0] + at[u].h * ss[1] + j * ss[2];
        if constexpr (BITS == 4) {
            code[u].x = *reinterpret_cast<const uint32_t *>(from + 4 * l);
            const uint32_t w = *reinterpret_cast<const uint32_t *>(scale + (D == 128 ? 4 * (l & 1) : 0));
            s[u][0] = __uint_as_float(w << 16);
            s[u][1] = __uint_as_float(w & 0xffff0000u);
        } else {
            code[u] = *reinterpret_cast<const uint2 *>(from + 8 * l);
            s[u][0] = *reinterpret_cast<const float *>(scale);
        }
    }
#pragma unroll
    for (int u = 0; u < QC_AHEAD; ++u) {
        if (!real[u]) continue;
        float y[8];
        values8<BITS>(y, code[u], s[u][0], s[u][1]);
        const long long *s3 = at[u].of_v ? p.vos : p.kos;
        Eight<T>::store(static_cast<T *>(at[u].of_v ? p.v_out : p.k_out) + at[u].b * s3[0] + at[u].h * s3[1] + at[u].i * s3[2] + 8 * l, y);
    }
}

}  // namespace obf
