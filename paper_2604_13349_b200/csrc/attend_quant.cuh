// Attention over a cache held in 8 or 4 bits.
//
// As for few rows over a bf16 cache, a block of four warps owns a tile of 8 NT query rows and a part of the keys, each warp walks
// its own stages of keys through a private ring of asynchronous copies, and keys lie on the M side of both products.  What multiplies are
// the codes: whole numbers of at most 8 bits are exact in 16-bit floating-point types, scales stay in fp32.
//
//   S_j = sum over the groups of k_scale_jg (sum over the group's channels of code_jc q_c)          codes and queries in fp16
//   O_c += sum over the keys of code_jc (p_j v_scale_jg(c))                                         codes and weights in bf16
//
// Queries are brought to a largest magnitude of 2^13 per row by a power of two, so fp16 holds a bf16 query to its last bit and an fp32
// query in two parts to 2^-22 of each number; weights, which reach over more powers of two than fp16 has, are bf16, in three parts for fp32
// outputs.  Fragments are made for codes in order: which channels (keys) a lane's part of a product stands for is free as long as both
// operands agree, so a lane takes whole words of a row and never moves a code to another lane.
#pragma once

#include <cuda_fp16.h>

#include "attend_few.cuh"
#include "quant_cache.cuh"

namespace obf {

template <int BITS, int D>
struct QuantStage {
    typedef QuantRow<BITS, D> Row;
    static constexpr int KEYS = Row::BYTES == 128 ? 16 : 32;
    static constexpr int CODES = KEYS * Row::BYTES, SCALES = KEYS * Row::SCALE_BYTES;
    static constexpr int BYTES = 2 * CODES + 2 * SCALES;               // K's codes, V's codes, K's scales, V's scales
    static constexpr int STAGES = BYTES > 4000 ? 3 : 4;
};

template <int BITS, int D, int ROWS>
__host__ __device__ constexpr size_t attend_quant_smem()
{
    const size_t ring = (size_t)AF_WARPS * QuantStage<BITS, D>::STAGES * QuantStage<BITS, D>::BYTES, end = few_finish_smem<D, ROWS>();
    return ring > end ? ring : end;
}

// Where 16-byte chunk c of a stage's key stands: rows of 32 and 64 bytes trade places and chunks so that a quarter of a warp's reads,
// of whole chunks of keys j and j + 4 (K), and a half's, of eight bytes of four neighbouring keys (V), meet every bank once.
template <int RB>
__device__ __forceinline__ uint32_t chunk_at(int key, int c)
{
    if constexpr (RB == 128) return key * 128 + (c ^ (2 * (key & 3)) ^ (key & 4)) * 16;
    if constexpr (RB == 64) {
        const int s = key ^ ((key >> 2) & 1);
        return s * 64 + (c ^ (s & 2)) * 16;
    }
    return (key ^ ((key >> 1) & 2)) * 32 + c * 16;
}

template <int N>
__device__ __forceinline__ void cp_async_small(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(N), "r"(real ? N : 0) : "memory");
}
__device__ __forceinline__ uint32_t lds1(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void lds(uint32_t (&v)[1], uint32_t a) { v[0] = lds1(a); }
__device__ __forceinline__ void lds(uint32_t (&v)[2], uint32_t a)
{
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(a) : "memory");
}
__device__ __forceinline__ void lds(uint32_t (&v)[4], uint32_t a)
{
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(a) : "memory");
}

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Codes as numbers.  Half n of a word's halves, four codes plus 8 each, as two fp16 numbers (1024 + u and 1024 + 16 u, less their offset)
// or as two bf16 numbers (128 + u, less 136): exact.
__device__ __forceinline__ uint32_t h2_sub(uint32_t x, float off)
{
    const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&x), __float2half2_rn(off));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ void nibbles_f16(uint32_t (&r)[4], uint32_t x)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t y = x >> (8 * i), lo = (y & 0x000f000fu) | 0x64006400u, hi = (y & 0x00f000f0u) | 0x64006400u;
        r[2 * i] = h2_sub(lo, 1032.f);
        const __half2 v = __hfma2(*reinterpret_cast<const __half2 *>(&hi), __float2half2_rn(0.0625f), __float2half2_rn(-72.f));
        r[2 * i + 1] = *reinterpret_cast<const uint32_t *>(&v);
    }
}
__device__ __forceinline__ uint32_t nibble_bf16(uint32_t x, int n)
{
    const uint32_t u = ((x >> (4 * n)) & 0x000f000fu) | 0x43004300u;
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&u), __float2bfloat162_rn(136.f));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// Four int8 codes as two pairs of fp16 numbers.
__device__ __forceinline__ void bytes_f16(uint32_t &lo, uint32_t &hi, uint32_t x)
{
    x ^= 0x80808080u;
    lo = h2_sub(__byte_perm(x, 0x64646464u, 0x4140), 1152.f);
    hi = h2_sub(__byte_perm(x, 0x64646464u, 0x4342), 1152.f);
}
// Byte n of two words (int8 codes plus 128) as a pair of bf16 numbers, by way of 2^23 + u.
__device__ __forceinline__ uint32_t byte_pair_bf16(uint32_t a, uint32_t b, int n)
{
    const float x = __uint_as_float(__byte_perm(a, 0x4b000000u, 0x7440 + n)), y = __uint_as_float(__byte_perm(b, 0x4b000000u, 0x7440 + n));
    return pack_bf16(x - 8388736.f, y - 8388736.f);
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Scales of a key, fp32.
template <int BITS, int D>
__device__ __forceinline__ void scales_of(float (&s)[QuantRow<BITS, D>::GROUPS], uint32_t a)
{
    if constexpr (BITS == 8) {
        s[0] = __uint_as_float(lds1(a));
    } else {
        uint32_t w[D / 64];
        lds(w, a);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) { s[2 * i] = bf16_lo(w[i]); s[2 * i + 1] = bf16_hi(w[i]); }
    }
}

// A pair of weights as bf16 numbers, in as many parts as the outputs' type needs (their sum is the weight but for the last part's rounding).
template <int PARTS>
__device__ __forceinline__ void split_weights(uint32_t (&r)[PARTS], float x, float y)
{
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        r[i] = pack_bf16(x, y);
        if (i + 1 < PARTS) { x -= bf16_lo(r[i]); y -= bf16_hi(r[i]); }
    }
}

template <typename TIN, int BITS, int D, int NT, bool CLUSTER>
__global__ void __launch_bounds__(AF_NT) k_attend_quant(const __grid_constant__ AttendDev p, const __grid_constant__ QuantDev c)
{
    extern __shared__ __align__(128) unsigned char aq_sm[];
    typedef QuantStage<BITS, D> Stage;
    typedef QuantRow<BITS, D> Row;
    constexpr int KS = D / 16, ROWS = 8 * NT, ST = Stage::STAGES, KEYS = Stage::KEYS, RB = Row::BYTES, CH = RB / 16, LR = 32 / CH, SB = Row::SCALE_BYTES, GR = Row::GROUPS;
    constexpr int PARTS = sizeof(TIN) == 4 ? 2 : 1;       // of a query
    constexpr int WPARTS = sizeof(TIN) == 4 ? 3 : 1;      // of a weight
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0) attend_status(p);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
    const int rows_seq = p.n_q * p.G, tiles = (rows_seq + ROWS - 1) / ROWS, parts = p.slots;
    unsigned x = blockIdx.x;
    const int part = x % parts;
    x /= parts;
    const int tile = x % tiles;
    x /= tiles;
    const int h = x % p.kv_heads, b = x / p.kv_heads;
    const int len = attend_len(p, b), ql = attend_q_len(p, b);

    KeyRange kr = {0, 0, 0};
    const int i0 = tile * ROWS / p.G, i1 = min((min((tile + 1) * ROWS, rows_seq) - 1) / p.G, ql - 1);
    if (i0 <= i1) kr = attend_range(p, len - ql + i0, len - ql + i1, len);
    const int n = kr.count(), per = ((n + 63) / 64 + parts - 1) / parts * 64;
    const int v0 = min((long long)part * per, (long long)n), v1 = min(v0 + per, n);

    const uint8_t *kb = c.k + b * c.ks[0] + h * c.ks[1], *vb = c.v + b * c.vs[0] + h * c.vs[1];
    const uint8_t *ksb = c.k_scale + b * c.kss[0] + h * c.kss[1], *vsb = c.v_scale + b * c.vss[0] + h * c.vss[1];

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(aq_sm) + warp * ST * Stage::BYTES;
    const int lc = lane % CH, lr = lane / CH;
    const int mine = (v1 - v0 + KEYS - 1) / KEYS;         // the part's stages, of which this warp does warp, warp + 4, ...
    auto fetch = [&](int st, int slot) {
        if (st < mine) {
            const uint32_t kd = ring + slot * Stage::BYTES, vd = kd + Stage::CODES, sd = vd + Stage::CODES;
            const int va = v0 + st * KEYS;
#pragma unroll
            for (int i = 0; i < KEYS / LR; ++i) {
                const int r = lr + i * LR, v = va + r;
                const bool real = v < v1;
                const long long j = kr.key(real ? v : v0);
                const uint32_t at = chunk_at<RB>(r, lc);
                cp_async16(kd + at, kb + j * c.ks[2] + lc * 16, real);
                cp_async16(vd + at, vb + j * c.vs[2] + lc * 16, real);
            }
            if (lane < KEYS) {
                const int v = va + lane;
                const bool real = v < v1;                 // (behind the part: zeros, whatever the cache holds there)
                const long long j = kr.key(real ? v : v0);
                cp_async_small<SB>(sd + lane * SB, ksb + j * c.kss[2], real);
                cp_async_small<SB>(sd + Stage::SCALES + lane * SB, vsb + j * c.vss[2], real);
            }
        }
        cp_commit();
    };
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) fetch(warp + s * AF_WARPS, s);

    // Queries as B fragments: of row 8 nt + lane / 4 a lane holds a quarter of the channels, those of its words of a key.
    uint32_t qf[PARTS][NT][KS][2];
    float row_c[NT][2];                                   // what makes logits (log2) of a product's rows 8 nt + 2 (lane mod 4) + e
    int row_t[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = tile * ROWS + nt * 8 + g8, i = r / p.G, g = r - i * p.G;
        const bool real = r < rows_seq && i < ql;
        const TIN *src = static_cast<const TIN *>(p.q) + b * p.qs[0] + (long long)(h * p.G + g) * p.qs[1] + (long long)i * p.qs[2];
        float q[D / 4];
        uint32_t top = 0;
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {                // eight channels at a time
            const int ch = BITS == 8 && D == 128 ? 16 * t4 + 8 * (w & 1) + 64 * (w >> 1) : t4 * (D / 4) + 8 * w;
            float y[8];
            if (real) {
                Eight<TIN> e;
                e.load(src + ch);
                e.get(y);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                q[8 * w + k] = real ? y[k] : 0.f;
                top = max(top, __float_as_uint(q[8 * w + k]) & 0x7fffffffu);
            }
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = min(max((int)(top >> 23), 27), 254);             // exponent of the largest, at least that of 2^-100
        const float up = __uint_as_float((uint32_t)(267 - e) << 23), down = __uint_as_float((uint32_t)(e - 13) << 23);
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                // the pair's two channels among the lane's
                const int a = BITS == 8 ? 4 * k + 2 * u : 2 * k + u, a2 = BITS == 8 ? a + 1 : a + D / 8;
                float y = q[a] * up, z = q[a2] * up;
#pragma unroll
                for (int part_q = 0; part_q < PARTS; ++part_q) {
                    const __half2 v = __floats2half2_rn(y, z);
                    qf[part_q][nt][k][u] = *reinterpret_cast<const uint32_t *>(&v);
                    y -= __low2float(v);
                    z -= __high2float(v);
                }
            }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            row_c[nt][u] = p.c * __shfl_sync(0xffffffffu, down, 4 * (2 * t4 + u));
            const int r2 = tile * ROWS + nt * 8 + 2 * t4 + u, i2 = r2 / p.G;
            row_t[nt][u] = r2 < rows_seq && i2 < ql ? len - ql + i2 : INT_MIN;
        }
    }

    float o[NT][KS][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) { m[nt][e] = -INFINITY; l[nt][e] = 0.f; }
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][k][e] = 0.f;
    }
    const bool one_t = p.n_q == 1;                        // every row of the tile sees every key of the range
    // Row r of a 16-key product stands for key  r / 2 + 4 (r mod 2)  of its half of eight: a lane then reads four neighbouring keys' values.
    const int key_s = (g8 >> 1) + 4 * (g8 & 1);
    int slot = 0;
    for (int st = warp; st < mine; st += AF_WARPS) {
        cp_wait<ST - 2>();
        __syncwarp();
        fetch(st + (ST - 1) * AF_WARPS, slot == 0 ? ST - 1 : slot - 1);
#pragma unroll
        for (int sub = 0; sub < KEYS / 16; ++sub) {
            const uint32_t kd = ring + slot * Stage::BYTES + sub * 16 * RB, vd = kd + Stage::CODES;
            const uint32_t sd = ring + slot * Stage::BYTES + 2 * Stage::CODES + (sub * 16 + key_s) * SB;
            float s[NT][4];
            // ---- logits ----
            {
                float k0[GR], k1[GR];
                scales_of<BITS, D>(k0, sd);
                scales_of<BITS, D>(k1, sd + 8 * SB);
                if constexpr (BITS == 4) {
                    constexpr int W = D / 32;             // words of a lane
                    uint32_t w0[W], w1[W];
                    if constexpr (D == 128) {
                        lds(w0, kd + chunk_at<RB>(key_s, t4));
                        lds(w1, kd + chunk_at<RB>(key_s + 8, t4));
                    } else {
                        lds(w0, kd + chunk_at<RB>(key_s, t4 >> 1) + (t4 & 1) * 8);
                        lds(w1, kd + chunk_at<RB>(key_s + 8, t4 >> 1) + (t4 & 1) * 8);
                    }
#pragma unroll
                    for (int j = 0; j < GR; ++j) {
                        const int sel = j & 1 ? 0x7632 : 0x5410;
                        uint32_t n0[4], n1[4];
                        nibbles_f16(n0, __byte_perm(w0[j >> 1], w0[(j >> 1) + W / 2], sel));
                        nibbles_f16(n1, __byte_perm(w1[j >> 1], w1[(j >> 1) + W / 2], sel));
                        float acc[NT][4];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[nt][e] = 0.f;
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const uint32_t a[4] = {n0[2 * i], n1[2 * i], n0[2 * i + 1], n1[2 * i + 1]};
#pragma unroll
                                for (int part_q = PARTS - 1; part_q >= 0; --part_q) mma_f16(acc[nt], a, qf[part_q][nt][2 * j + i][0], qf[part_q][nt][2 * j + i][1]);
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float y = acc[nt][e] * (e < 2 ? k0[j] : k1[j]);
                                s[nt][e] = j == 0 ? y : s[nt][e] + y;
                            }
                        }
                    }
                } else {
                    uint32_t w0[KS], w1[KS];
#pragma unroll
                    for (int half = 0; half < KS / 4; ++half) {
                        uint32_t u0[4], u1[4];
                        lds(u0, kd + chunk_at<RB>(key_s, t4 + 4 * half));
                        lds(u1, kd + chunk_at<RB>(key_s + 8, t4 + 4 * half));
#pragma unroll
                        for (int i = 0; i < 4; ++i) { w0[4 * half + i] = u0[i]; w1[4 * half + i] = u1[i]; }
                    }
                    float acc[NT][2][4];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[nt][0][e] = acc[nt][1][e] = 0.f;
#pragma unroll
                    for (int k = 0; k < KS; ++k) {
                        uint32_t a[4];
                        bytes_f16(a[0], a[2], w0[k]);
                        bytes_f16(a[1], a[3], w1[k]);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int part_q = PARTS - 1; part_q >= 0; --part_q) mma_f16(acc[nt][k & 1], a, qf[part_q][nt][k][0], qf[part_q][nt][k][1]);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[nt][e] = (acc[nt][0][e] + acc[nt][1][e]) * (e < 2 ? k0[0] : k1[0]);
                }
            }
            // ---- weights: s[nt][2 u + e] is key 8 u + key_s of the sixteen, row 8 nt + 2 (lane mod 4) + e ----
            const int va = v0 + st * KEYS + sub * 16 + key_s;
            bool raise = false;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int v = va + 8 * u, j = kr.key(v);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const bool sees = v < v1 && (one_t || attend_sees(p, row_t[nt][e], j));
                        float &y = s[nt][2 * u + e];
                        y = sees ? y * row_c[nt][e] : -INFINITY;
                        raise = raise || y > m[nt][e] + AF_RAISE;
                    }
            }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(fmaxf(s[nt][e], s[nt][2 + e]), m[nt][e]);
#pragma unroll
                        for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                        const float f = mx == -INFINITY ? 1.f : ex2(m[nt][e] - mx);
                        m[nt][e] = mx;
                        l[nt][e] *= f;
#pragma unroll
                        for (int k = 0; k < KS; ++k) { o[nt][k][e] *= f; o[nt][k][2 + e] *= f; }
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float r0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], r1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    s[nt][2 * u] = ex2(s[nt][2 * u] - r0);
                    s[nt][2 * u + 1] = ex2(s[nt][2 * u + 1] - r1);
                    l[nt][0] += s[nt][2 * u];
                    l[nt][1] += s[nt][2 * u + 1];
                }
            }
            // ---- values ----
            float k0[GR], k1[GR];
            scales_of<BITS, D>(k0, sd + Stage::SCALES);
            scales_of<BITS, D>(k1, sd + Stage::SCALES + 8 * SB);
            constexpr int W = RB / 32;                    // words of a lane
            uint32_t w[4][W];                             // of keys lane mod 4 + 4 i
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = t4 + 4 * i;
                if constexpr (W == 4) lds(w[i], vd + chunk_at<RB>(key, g8));
                else if constexpr (W == 2) lds(w[i], vd + chunk_at<RB>(key, g8 >> 1) + (g8 & 1) * 8);
                else lds(w[i], vd + chunk_at<RB>(key, g8 >> 2) + (g8 & 3) * 4);
                if constexpr (BITS == 8) {
#pragma unroll
                    for (int q = 0; q < W; ++q) w[i][q] ^= 0x80808080u;
                }
            }
#pragma unroll
            for (int j = 0; j < GR; ++j) {
                uint32_t pf[NT][WPARTS][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float f = u ? k1[j] : k0[j];
                        uint32_t pw[WPARTS];
                        split_weights<WPARTS>(pw, s[nt][2 * u] * f, s[nt][2 * u + 1] * f);
#pragma unroll
                        for (int q = 0; q < WPARTS; ++q) pf[nt][q][u] = transpose8x8(pw[q]);
                    }
                constexpr int MT = KS / GR;               // channel tiles of the group
                if constexpr (BITS == 4) {
                    const int sel = j & 1 ? 0x7632 : 0x5410;
                    const uint32_t ab = __byte_perm(w[0][j >> 1], w[1][j >> 1], sel), cd = __byte_perm(w[2][j >> 1], w[3][j >> 1], sel);
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        const uint32_t a[4] = {nibble_bf16(ab, 2 * i), nibble_bf16(ab, 2 * i + 1), nibble_bf16(cd, 2 * i), nibble_bf16(cd, 2 * i + 1)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int q = WPARTS - 1; q >= 0; --q) mma_bf16(o[nt][2 * j + i], a, pf[nt][q][0], pf[nt][q][1]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        const int q0 = i >> 1, n0 = 2 * (i & 1);
                        const uint32_t a[4] = {byte_pair_bf16(w[0][q0], w[1][q0], n0), byte_pair_bf16(w[0][q0], w[1][q0], n0 + 1),
                                               byte_pair_bf16(w[2][q0], w[3][q0], n0), byte_pair_bf16(w[2][q0], w[3][q0], n0 + 1)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int q = WPARTS - 1; q >= 0; --q) mma_bf16(o[nt][i], a, pf[nt][q][0], pf[nt][q][1]);
                    }
                }
            }
        }
        slot = slot + 1 == ST ? 0 : slot + 1;
    }
    cp_wait<0>();
    __syncthreads();

    // the warps' results: O as [warp][row][D + 4], then references and sums; tile k of O holds channels (lane / 4) D / 8 + 2 k, + 1
    constexpr int LD = D + 4;
    float *osm = reinterpret_cast<float *>(aq_sm), *ml = osm + AF_WARPS * ROWS * LD;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float z = l[nt][e];
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) z += __shfl_xor_sync(0xffffffffu, z, w);
            const int row = 8 * nt + 2 * t4 + e;
            if (lane < 4) { ml[(warp * ROWS + row) * 2] = m[nt][e]; ml[(warp * ROWS + row) * 2 + 1] = z; }
#pragma unroll
            for (int k = 0; k < KS; k += 2)
                *reinterpret_cast<float4 *>(&osm[(warp * ROWS + row) * LD + g8 * (D / 8) + 2 * k]) = make_float4(o[nt][k][e], o[nt][k][2 + e], o[nt][k + 1][e], o[nt][k + 1][2 + e]);
        }
    __syncthreads();
    few_finish<TIN, D, ROWS, false, CLUSTER>(p, osm, ml, tile, part, parts, rows_seq, rows_seq, h, b, len, ql, kr, v0, v1);
}

}  // namespace obf
