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
    // Reading for attention: what the queries (q_lens, or n_q of each sequence) see through a window, and behind it the first tokens;
    // of 8 bits the codes, with factors (AttendDev) apart.
    const int32_t *q_lens;
    int32_t n_q, window, sinks;
    float *factors;
    long long factor_stride;
    float c;                               // of K's factors
    FastDiv by_rows, by_heads;
};

constexpr int QC_NT = 256;

// Scale of numbers whose largest magnitude has the bits `top` (as integers, so that what is not a number counts as the largest): not a
// number where one of them is not finite, zero where all are below 2^-110, whose scale would lose bits.
__device__ __forceinline__ float scale8(uint32_t top)
{
    const float s = __fdiv_rn(__uint_as_float(top), 127.f);
    return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : top < (127u - 110u) << 23 ? 0.f : s;
}
// max / 7 rounded half to even to five bits.  Of a bf16 maximum the product with 1 / 7, rounded to 17 bits first, will do: the quotient is halfway
// between two numbers of five bits or at least 2^-12 of itself away from there.
template <typename T>
__device__ __forceinline__ float scale4(uint32_t top)
{
    const float x = __uint_as_float(top);
    uint32_t i;
    if constexpr (sizeof(T) == 4) i = __float_as_uint(__fdiv_rn(x, 7.f));
    else i = (__float_as_uint(x * (1.f / 7.f)) + 0x40u) & ~0x7fu;
    const float s = __uint_as_float((i + 0x3ffffu + ((i >> 19) & 1u)) & 0xfff80000u);
    return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : top < (127u - 110u) << 23 ? 0.f : s;
}

// Codes as the low bits of fp32 numbers near 1.5 * 2^23, where a sum is rounded to a whole number, half to even.
constexpr float QC_ONES = 12582912.f;

// x / scale in 4 bits, plus QC_ONES + 8.  bf16 numbers over a scale of five bits: the quotient is n + 1/2 exactly or at least 1/496 away from it
// (2 x and (2 n + 1) scale are multiples of an eighth of the scale's last bit), so rounding the product to a multiple of 2^-10 (at
// 1.5 * 2^13) first undoes its error of 2^-20.  fp32 numbers: the product tells, or where it is too near to n + 1/2 for that, the quotient.
template <typename T>
__device__ __forceinline__ float code4(float x, float scale, float inv)
{
    if constexpr (sizeof(T) == 2) {
        constexpr float GRID = 12288.f;
        return __fadd_rn(__fmaf_rn(x, inv, GRID), QC_ONES + 8.f - GRID);
    } else {
        const float t = __fmaf_rn(x, inv, QC_ONES + 8.f), d = __fmaf_rn(x, inv, -(t - (QC_ONES + 8.f)));
        return fabsf(d) > 0.49995f ? __fadd_rn(__fdiv_rn(x, scale), QC_ONES + 8.f) : t;
    }
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
    __device__ __forceinline__ void store(T *p) const
    {
        constexpr int N = sizeof(T) == 4 ? 2 : 1;
#pragma unroll
        for (int i = 0; i < N; ++i) reinterpret_cast<uint4 *>(p)[i] = w[i];
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                w[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
        } else {
            w[0] = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        }
    }
};

// 32 bytes, a sector of memory, in one store where the address allows it (callers promise 16): reading back 16 caches of 3001 to 8192 rows in 4 bits takes
// 74 us with it, 97 us with two stores of 16 bytes.
__device__ __forceinline__ void store32(void *p, const uint4 &a, const uint4 &b)
{
    if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
    } else {
        static_cast<uint4 *>(p)[0] = a;
        static_cast<uint4 *>(p)[1] = b;
    }
}

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

// Where a row of a call is read and written.  Rows of one head lie `step` apart.
struct RowPlace {
    const char *in;                        // rows to write / rows of the cache's codes
    const uint8_t *in_scale;               // reading
    uint8_t *code, *scale;                 // writing
    char *out;                             // values
    float *factor, c;                      // reading codes: where the scale goes, times what
};

__device__ __forceinline__ const char *row_ptr(const void *base, const long long *st, const RowAt &at, long long row, int size)
{
    return static_cast<const char *>(base) + (at.b * st[0] + at.h * st[1] + row * st[2]) * size;
}

// Sixteen neighbouring channels of a row, as loaded.
template <typename T>
struct Sixteen {
    Eight<T> half[2];
    __device__ __forceinline__ void load(const T *p)
    {
        half[0].load(p);
        half[1].load(p + 8);
    }
    __device__ __forceinline__ void store(T *p) const
    {
        if constexpr (sizeof(T) == 2) {
            store32(p, half[0].w[0], half[1].w[0]);
        } else {
            store32(p, half[0].w[0], half[0].w[1]);
            store32(p + 8, half[1].w[0], half[1].w[1]);
        }
    }
};

// Largest magnitudes of the four groups that sixteen channels in 4 bits belong to (four neighbours each), as bits.
template <typename T>
__device__ __forceinline__ void tops4(uint32_t (&top)[4], const Sixteen<T> &in, int lanes)
{
    if constexpr (sizeof(T) == 2) {
        // two groups in a word: bf16 magnitudes compare as 16-bit numbers
        uint32_t two[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 w = in.half[i].w[0];
            const uint32_t a = __vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), b = __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu);
            two[i] = __vmaxu2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
        }
        if (lanes == 4) two[0] = two[1] = __vmaxu2(two[0], two[1]);            // heads of 64 channels have two groups
#pragma unroll
        for (int w = 1; w < 8; w <<= 1) {
            if (w >= lanes) continue;
            two[0] = __vmaxu2(two[0], __shfl_xor_sync(0xffffffffu, two[0], w));
            if (lanes == 8) two[1] = __vmaxu2(two[1], __shfl_xor_sync(0xffffffffu, two[1], w));
        }
        if (lanes == 4) two[1] = two[0];
#pragma unroll
        for (int i = 0; i < 2; ++i) { top[2 * i] = two[i] << 16; top[2 * i + 1] = two[i] & 0xffff0000u; }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 w = in.half[i / 2].w[i % 2];
            top[i] = max(max(w.x & 0x7fffffffu, w.y & 0x7fffffffu), max(w.z & 0x7fffffffu, w.w & 0x7fffffffu));
        }
        if (lanes == 4) { top[0] = top[2] = max(top[0], top[2]); top[1] = top[3] = max(top[1], top[3]); }
#pragma unroll
        for (int w = 1; w < 8; w <<= 1) {
            if (w >= lanes) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) top[i] = max(top[i], __shfl_xor_sync(0xffffffffu, top[i], w));
        }
    }
}

// Largest magnitude of sixteen channels, as bits.
template <typename T>
__device__ __forceinline__ uint32_t top8(const Sixteen<T> &in)
{
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
            const uint4 w = in.half[i].w[k];
            if constexpr (sizeof(T) == 2)
                top = __vmaxu2(top, __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu)));
            else
                top = max(top, max(max(w.x & 0x7fffffffu, w.y & 0x7fffffffu), max(w.z & 0x7fffffffu, w.w & 0x7fffffffu)));
        }
    return sizeof(T) == 2 ? max(top << 16, top & 0xffff0000u) : top;
}

// Rows of a thread in flight, and blocks of a multiprocessor (bf16 rows to 4 bits: 4 rows 81 us, 2 rows 84; to 8 bits 88 and 74).
template <typename T, int BITS>
constexpr int QW_AHEAD = sizeof(T) == 2 && BITS == 4 ? 4 : 2;
template <typename T, int BITS>
constexpr int QW_BLOCKS = sizeof(T) == 2 && BITS == 8 ? 4 : 3;

// Writing: D / 16 lanes a row, sixteen channels each; a thread's rows are all read before the first of them is worked on.  Blocks whose rows are
// all one head's have their places in common.  Where there are many rows it is bound by the instructions that form codes about as much as by HBM (8 prompts of
// 3001 to 8192 rows to 4 bits, with values 79 us, 5.3 TB/s; 36 x 1012 rows to 8 bits, with values 73 us, 5.2 TB/s), by the latency of a launch and two
// dependent reads where there are few.
template <typename T, int BITS, int D, bool VALUES, bool ONE>
__device__ __forceinline__ void quant_write(const RowsDev &p, const QuantDev &c, const RowAt &head)
{
    constexpr int L = D / 16, R = QC_NT / L, AHEAD = QW_AHEAD<T, BITS>;       // lanes of a row, rows of a block at a time
    const int l = threadIdx.x % L;
    Sixteen<T> in[AHEAD];
    RowPlace at[AHEAD];
    bool real[AHEAD];
    const auto first_row = [&](int b) {                   // row of the cache that the sequence's first new row goes to
        const int n_new = p.new_lens ? min(max(p.new_lens[b], 0), p.rows) : p.rows;
        return make_int2(n_new, (p.lens ? min(max(p.lens[b], -(1 << 30)), 1 << 30) : n_new) - n_new);
    };
    const auto place = [&](const RowAt &r, int to) {
        RowPlace q;
        q.in = row_ptr(r.of_v ? p.v : p.k, r.of_v ? p.vs : p.ks, r, r.i, sizeof(T)) + 16 * l * sizeof(T);
        q.code = reinterpret_cast<uint8_t *>(const_cast<char *>(row_ptr(r.of_v ? c.v : c.k, r.of_v ? c.vs : c.ks, r, to, 1)));
        q.scale = reinterpret_cast<uint8_t *>(const_cast<char *>(row_ptr(r.of_v ? c.v_scale : c.k_scale, r.of_v ? c.vss : c.kss, r, to, 1)));
        if constexpr (VALUES) q.out = const_cast<char *>(row_ptr(r.of_v ? p.v_out : p.k_out, r.of_v ? p.vos : p.kos, r, r.i, sizeof(T))) + 16 * l * sizeof(T);
        return q;
    };
    if constexpr (ONE) {
        const int2 new_at = first_row(head.b);
        RowAt r = head;
        r.i += threadIdx.x / L;
        const RowPlace q = place(r, (int)r.i + new_at.y);
        const long long in = (head.of_v ? p.vs : p.ks)[2] * (long long)sizeof(T) * R, code = (head.of_v ? c.vs : c.ks)[2] * R, scale = (head.of_v ? c.vss : c.kss)[2] * R,
                        out = (head.of_v ? p.vos : p.kos)[2] * (long long)sizeof(T) * R;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = (int)r.i + u * R;
            real[u] = i < new_at.x && i + new_at.y >= 0 && i + new_at.y < p.capacity;
            at[u].in = q.in + u * in;
            at[u].code = q.code + u * code;
            at[u].scale = q.scale + u * scale;
            if constexpr (VALUES) at[u].out = q.out + u * out;
        }
    } else {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint32_t f = blockIdx.x * (R * AHEAD) + u * R + threadIdx.x / L;
            real[u] = f < p.total;
            if (!real[u]) continue;
            const RowAt r = row_at(p, f);
            const int2 new_at = first_row(r.b);
            const long long to = (long long)r.i + new_at.y;
            real[u] = (int)r.i < new_at.x && to >= 0 && to < p.capacity;
            at[u] = place(r, real[u] ? (int)to : 0);
        }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        in[u] = {};
        if (real[u]) in[u].load(reinterpret_cast<const T *>(at[u].in));
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        uint32_t top[4];
        if constexpr (BITS == 4) {
            tops4<T>(top, in[u], L);
        } else {
            top[0] = top8(in[u]);
#pragma unroll
            for (int w = 1; w < L; w <<= 1) top[0] = max(top[0], __shfl_xor_sync(0xffffffffu, top[0], w));
        }
        float s[4], inv[4];
        if constexpr (BITS == 4) {
            // each lane works one group's scale out and passes it on
            const float own = scale4<T>(l & 2 ? (l & 1 ? top[3] : top[2]) : (l & 1 ? top[1] : top[0]));
            const float own_inv = own > 0.f ? __frcp_rn(own) : 0.f;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                s[g] = __shfl_sync(0xffffffffu, own, g, 4);
                inv[g] = __shfl_sync(0xffffffffu, own_inv, g, 4);
            }
        } else {
            s[0] = scale8(top[0]);
            inv[0] = s[0] > 0.f ? __frcp_rn(s[0]) : 0.f;
        }
        if (!real[u]) continue;
        // a scale that is not a number: codes of zero, whatever the channels hold
        bool whole = s[0] == s[0];
        if constexpr (BITS == 4) whole = whole && s[1] == s[1] && s[2] == s[2] && s[3] == s[3];
        uint32_t word[4];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float x[8], y[8];
            in[u].half[half].get(x);
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float f = s[BITS == 4 ? 2 * half + i / 4 : 0];
                    if (f != f) x[i] = 0.f;
                }
            }
            if constexpr (BITS == 4) {
                uint32_t w = 0u;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int g = 2 * half + i / 4;
                    const float t = code4<T>(x[i], s[g], inv[g]);
                    w = (__float_as_uint(t) << (4 * i)) + w;
                    y[i] = (t - (QC_ONES + 8.f)) * s[g];
                }
                word[half] = w - 0x4b400000u * 0x11111111u;      // (modulo 2^32: what the places of 1.5 * 2^23 add up to)
            } else {
                float t[8], worst = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    t[i] = __fmaf_rn(x[i], inv[0], QC_ONES);
                    worst = fmaxf(worst, fabsf(__fmaf_rn(x[i], inv[0], QC_ONES - t[i])));
                }
                // The code is the whole number nearest to the fp32 quotient, which the product is within 1.2e-5 of (|x / scale| <= 127): only
                // where one is nearer than that to n + 1/2 the quotients are formed.
                if (worst > 0.49998f && s[0] > 0.f) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (fabsf(__fmaf_rn(x[i], inv[0], QC_ONES - t[i])) > 0.49998f) t[i] = __fadd_rn(__fdiv_rn(x[i], s[0]), QC_ONES);
                }
                uint32_t b[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    b[i] = __float_as_uint(t[i]);
                    y[i] = (t[i] - QC_ONES) * s[0];
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    word[2 * half + i] = __byte_perm(__byte_perm(b[4 * i], b[4 * i + 1], 0x0040), __byte_perm(b[4 * i + 2], b[4 * i + 3], 0x0040), 0x5410);
            }
            if constexpr (VALUES) {
                Eight<T> v;
                v.set(y);
                v.store(reinterpret_cast<T *>(at[u].out) + 8 * half);
            }
        }
        if constexpr (BITS == 4) {
            *reinterpret_cast<uint2 *>(at[u].code + 8 * l) = make_uint2(word[0], word[1]);
            const uint32_t s01 = __float_as_uint(s[0]) >> 16 | (__float_as_uint(s[1]) & 0xffff0000u), s23 = __float_as_uint(s[2]) >> 16 | (__float_as_uint(s[3]) & 0xffff0000u);
            if (l == 0) {
                if constexpr (D == 128) *reinterpret_cast<uint2 *>(at[u].scale) = make_uint2(s01, s23);
                else *reinterpret_cast<uint32_t *>(at[u].scale) = s01;
            }
        } else {
            *reinterpret_cast<uint4 *>(at[u].code + 16 * l) = make_uint4(word[0], word[1], word[2], word[3]);
            if (l == 0) *reinterpret_cast<float *>(at[u].scale) = s[0];
        }
    }
}

template <typename T, int BITS, int D, bool VALUES>
__global__ void __launch_bounds__(QC_NT, (QW_BLOCKS<T, BITS>)) k_quant_write(const __grid_constant__ RowsDev p, const __grid_constant__ QuantDev c)
{
    pdl_wait();
    pdl_trigger();
    constexpr uint32_t ROWS = QC_NT / (D / 16) * QW_AHEAD<T, BITS>;
    const RowAt head = row_at(p, blockIdx.x * ROWS);
    if (head.i + ROWS <= (uint32_t)p.rows) quant_write<T, BITS, D, VALUES, true>(p, c, head);
    else quant_write<T, BITS, D, VALUES, false>(p, c, head);
}

// Eight neighbouring channels' values from their codes (a word, two words) and scales (two bf16 ones in a word, one).
template <typename T, int BITS>
__device__ __forceinline__ void values8(Eight<T> &dst, uint2 code, uint32_t scale)
{
    if constexpr (BITS == 4 && sizeof(T) == 2) {
        // Four codes of either half of the word side by side as 128 + u, less 136, times the halves' scales: one rounding, of the product.
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t u = ((code.x >> (4 * i)) & 0x000f000fu) | 0x43004300u;
            const __nv_bfloat162 v = __hmul2(__hadd2(*reinterpret_cast<__nv_bfloat162 *>(&u), __float2bfloat162_rn(-136.f)), *reinterpret_cast<const __nv_bfloat162 *>(&scale));
            r[i] = *reinterpret_cast<const uint32_t *>(&v);
        }
        dst.w[0] = make_uint4(__byte_perm(r[0], r[1], 0x5410), __byte_perm(r[2], r[3], 0x5410), __byte_perm(r[0], r[1], 0x7632), __byte_perm(r[2], r[3], 0x7632));
    } else {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // codes plus an offset as the last bits of 2^23 + u
            if constexpr (BITS == 4) {
                y[i] = (__uint_as_float(((code.x >> (4 * i)) & 15u) | 0x4b000000u) - 8388616.f) * (i < 4 ? __uint_as_float(scale << 16) : __uint_as_float(scale & 0xffff0000u));
            } else {
                y[i] = (__uint_as_float(__byte_perm((i < 4 ? code.x : code.y) ^ 0x80808080u, 0x4b000000u, 0x7440 + i % 4)) - 8388736.f) * __uint_as_float(scale);
            }
        }
        dst.set(y);
    }
}

// Reading rows first .. first + rows - 1 back, laid out as for writing: sixteen channels a lane, a sector in bf16.  Bound by HBM (16 caches of 3001 to 8192
// rows in 4 bits: 74 us, 6.3 TB/s; eight channels a lane, stores of 16 bytes next to one another: 82 us).
constexpr int QR_AHEAD = 4;

template <typename T, int BITS, int D, bool CODES, bool ONE>
__device__ __forceinline__ void quant_read(const RowsDev &p, const QuantDev &c, const RowAt &head)
{
    constexpr int L = D / 16, R = QC_NT / L;
    const int l = threadIdx.x % L;
    uint4 code[QR_AHEAD];
    uint32_t s[QR_AHEAD][2];
    RowPlace at[QR_AHEAD];
    bool real[QR_AHEAD];
    // rows x .. y - 1 and the first sinks are read
    const auto rows_of = [&](int b) {
        const int n = p.lens ? min(p.lens[b], p.capacity) : p.capacity;
        int lo = 0;
        if (p.window) lo = max(0, n - (p.q_lens ? min(max(p.q_lens[b], 0), p.n_q) : p.n_q) - p.window + 1) & ~3;
        return make_int2(lo, n);
    };
    const auto is_read = [&](int2 range, int j) { return j < range.y && (j >= range.x || j < p.sinks); };
    const auto place = [&](const RowAt &r) {
        RowPlace q;
        q.in = row_ptr(r.of_v ? c.v : c.k, r.of_v ? c.vs : c.ks, r, p.first + (long long)r.i, 1) + 2 * BITS * l;
        q.in_scale = reinterpret_cast<const uint8_t *>(row_ptr(r.of_v ? c.v_scale : c.k_scale, r.of_v ? c.vss : c.kss, r, p.first + (long long)r.i, 1));
        q.out = const_cast<char *>(row_ptr(r.of_v ? p.v_out : p.k_out, r.of_v ? p.vos : p.kos, r, r.i, sizeof(T))) + 16 * l * sizeof(T);
        if constexpr (CODES) {
            // two keys' factors of logits, two of weights (rows of a thread lie multiples of two apart)
            q.factor = p.factors + (((long long)r.b * p.by_heads.d + r.h) * p.factor_stride + (r.i & ~1u)) * 2 + (r.of_v ? 2 : 0) + (r.i & 1u);
            q.c = r.of_v ? 1.f : p.c;
        }
        return q;
    };
    if constexpr (ONE) {
        const int2 range = rows_of(head.b);
        RowAt r = head;
        r.i += threadIdx.x / L;
        const RowPlace q = place(r);
        const long long in = (head.of_v ? c.vs : c.ks)[2] * R, scale = (head.of_v ? c.vss : c.kss)[2] * R, out = (head.of_v ? p.vos : p.kos)[2] * (long long)sizeof(T) * R;
#pragma unroll
        for (int u = 0; u < QR_AHEAD; ++u) {
            real[u] = is_read(range, p.first + (int)r.i + u * R);
            at[u].in = q.in + u * in;
            at[u].in_scale = q.in_scale + u * scale;
            at[u].out = q.out + u * out;
            if constexpr (CODES) { at[u].factor = q.factor + 2 * u * R; at[u].c = q.c; }
        }
    } else {
#pragma unroll
        for (int u = 0; u < QR_AHEAD; ++u) {
            const uint32_t f = blockIdx.x * (R * QR_AHEAD) + u * R + threadIdx.x / L;
            real[u] = f < p.total;
            if (!real[u]) continue;
            const RowAt r = row_at(p, f);
            real[u] = is_read(rows_of(r.b), p.first + (int)r.i);
            at[u] = place(r);
        }
    }
#pragma unroll
    for (int u = 0; u < QR_AHEAD; ++u) {
        if (!real[u]) continue;
        if constexpr (BITS == 4) {
            const uint2 w = *reinterpret_cast<const uint2 *>(at[u].in);
            code[u].x = w.x;
            code[u].z = w.y;
        } else {
            code[u] = *reinterpret_cast<const uint4 *>(at[u].in);
        }
        s[u][0] = s[u][1] = *reinterpret_cast<const uint32_t *>(at[u].in_scale);
        if constexpr (BITS == 4 && D == 128) s[u][1] = *reinterpret_cast<const uint32_t *>(at[u].in_scale + 4);
    }
#pragma unroll
    for (int u = 0; u < QR_AHEAD; ++u) {
        if (!real[u]) continue;
        Sixteen<T> row;
        values8<T, BITS>(row.half[0], make_uint2(code[u].x, code[u].y), CODES ? 0x3f800000u : s[u][0]);
        values8<T, BITS>(row.half[1], make_uint2(code[u].z, code[u].w), CODES ? 0x3f800000u : s[u][1]);
        row.store(reinterpret_cast<T *>(at[u].out));
        if (CODES && l == 0) *at[u].factor = __uint_as_float(s[u][0]) * at[u].c;
    }
}

// CODES (8 bits): the codes themselves, as bf16 numbers, and the scales apart.
template <typename T, int BITS, int D, bool CODES>
__global__ void __launch_bounds__(QC_NT) k_quant_read(const __grid_constant__ RowsDev p, const __grid_constant__ QuantDev c)
{
    pdl_wait();
    pdl_trigger();
    constexpr uint32_t ROWS = QC_NT / (D / 16) * QR_AHEAD;
    const RowAt head = row_at(p, blockIdx.x * ROWS);
    if (head.i + ROWS <= (uint32_t)p.rows) quant_read<T, BITS, D, CODES, true>(p, c, head);
    else quant_read<T, BITS, D, CODES, false>(p, c, head);
}

}  // namespace obf
