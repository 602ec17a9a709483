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
// operands agree, so a lane takes whole words of a row and never moves a code to another lane.  A product's eight columns are eight query rows; their
// fragments stand in shared memory for all four warps, which leaves the registers to the output.
//
// Bound by instructions and their latencies in tiles of 16 rows and more: the matrix pipe is busy for 32 % (tiles of 16 rows in bf16) and 37 % (fp32, 24 rows), issue slots
// for 59 % and 54 %, with two blocks of four warps a multiprocessor, which wait most for their own last results.  16 sequences in 4 bits, us from a graph: 16, 20 and 64
// query rows a KV head 66, 90 and 190; fp32, 64 channels, 20 rows 80, where three weights' parts, two queries' and their sums of sixteen keys make 60 products of 8 cycles
// for sixteen keys.
#pragma once

#include <cuda_fp16.h>

#include "attend_few.cuh"
#include "quant_cache.cuh"

namespace obf {

constexpr float AQ_NONE = -3e38f;                         // reference of a row that has seen no key: any logit raises it
// The power of two of weights, added to a logit behind the subtraction of its reference (taken off the reference it would be lost from logits of 2^31 on).
// bf16 calls: 2^75 times as large, since what they multiply is in units of 2^-133.  fp32 calls: 2^-24 times, so that 2^20 keys that weigh 2^8 times as much
// as their reference stay within fp32's range with values of 2^107.
template <typename TIN>
constexpr float AQ_BIAS = sizeof(TIN) == 4 ? -24.f : 75.f;
// What brings a warp's sums of weights, and of weights times codes, to where they are joined: in bf16 out of the bias, the latter out of the codes' unit too (at once,
// since 2^75 times a value and a number of keys may be beyond fp32's range where their average is not); in fp32 nothing, the bias is left to the lse.
template <typename TIN>
constexpr float AQ_SUM = sizeof(TIN) == 4 ? 1.f : 0x1p-75f;
template <typename TIN>
constexpr float AQ_VALUE = sizeof(TIN) == 4 ? 1.f : 0x1p58f;
template <typename TIN>
constexpr float AQ_LSE = sizeof(TIN) == 4 ? 0x1p24f : 1.f;

template <typename TIN>
__device__ __forceinline__ float aq_weight(float s, float m) { return ex2(__fadd_rn(s - m, AQ_BIAS<TIN>)); }

template <int BITS, int D>
struct QuantStage {
    typedef QuantRow<BITS, D> Row;
    static constexpr int KEYS = Row::BYTES == 128 ? 16 : 32;
    static constexpr int CODES = KEYS * Row::BYTES, SCALES = KEYS * Row::SCALE_BYTES;
    static constexpr int BYTES = 2 * CODES + 2 * SCALES;               // K's codes, V's codes, K's scales, V's scales
    static constexpr int STAGES = BYTES > 4000 ? 2 : 3;
};

// Shared memory of a block: the rings, `more` behind them, over all of it at the end the warps' results.
template <int BITS, int D>
constexpr int AQ_RING = AF_WARPS * QuantStage<BITS, D>::STAGES * QuantStage<BITS, D>::BYTES;
template <int BITS, int D, int ROWS>
__host__ __device__ constexpr size_t attend_quant_smem(size_t more)
{
    const size_t ring = AQ_RING<BITS, D> + more, end = few_finish_smem<D, ROWS>();
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
__device__ __forceinline__ void cp_async_all(uint32_t dst, const void *src)
{
    if constexpr (N == 16) asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(N) : "memory");
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

// The same on top of zeros, which take no registers.
__device__ __forceinline__ void mma_f16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ void mma_bf16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// c += a * (the sum of the parts): on top of c, or, EXACT, by itself and then added, since matrix products cut off what their sums cannot hold, which
// over thousands of keys all goes one way.
template <bool EXACT, int PARTS>
__device__ __forceinline__ void mma_weights(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&w)[PARTS][2])
{
    if constexpr (EXACT) {
        float t[4];
        mma_bf16_first(t, a, w[PARTS - 1][0], w[PARTS - 1][1]);
#pragma unroll
        for (int q = PARTS - 2; q >= 0; --q) mma_bf16(t, a, w[q][0], w[q][1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] += t[e];
    } else {
#pragma unroll
        for (int q = PARTS - 1; q >= 0; --q) mma_bf16(c, a, w[q][0], w[q][1]);
    }
}

// Codes as numbers, without arithmetic: the bits of a small whole number u are the fp16 number u 2^-24 (u < 2048) and the bf16 number
// u 2^-133 (u < 256), and matrix products take such numbers exactly.  A word of two halves of four codes plus 8 gives, by masks,
// pairs of codes 0 and 2 and, sixteen times as large, of codes 1 and 3 of the halves.
__device__ __forceinline__ void nibbles(uint32_t (&r)[4], uint32_t x)
{
    r[0] = x & 0x000f000fu;
    r[1] = x & 0x00f000f0u;
    r[2] = (x >> 8) & 0x000f000fu;
    r[3] = (x >> 8) & 0x00f000f0u;
}
// Their offsets: of bf16 pairs, 8 in the first kind of place, 8 * 16 in the second, both; 128 of bytes.
constexpr uint32_t AQ_MINUS_8 = 0x80088008u, AQ_MINUS_128 = 0x80808080u, AQ_MINUS_136 = 0x80888088u;
__device__ __forceinline__ uint32_t add_bf16(uint32_t x, uint32_t y)
{
    uint32_t r;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}
// fp32 calls: such small numbers have few bits above the matrix product's sums, which align what they add by exponents as written, so codes become
// numbers of full size, their offsets taken off: 1024 + u, 1024 + 16 u in fp16, 128 + u in bf16, 2^23 + u of bytes on the way to bf16.
__device__ __forceinline__ uint32_t add_f16(uint32_t x, uint32_t y)
{
    uint32_t r;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}
constexpr uint32_t AQ_F16_8 = 0xe408e408u, AQ_F16_128 = 0xe480e480u;       // -1032, -1152 in fp16
__device__ __forceinline__ void nibbles_f16(uint32_t (&r)[4], uint32_t x)       // codes 1 and 3 sixteenfold
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t y = i < 2 ? x : x >> 8;
        r[i] = add_f16((i & 1 ? y & 0x00f000f0u : y & 0x000f000fu) | 0x64006400u, i & 1 ? AQ_F16_128 : AQ_F16_8);
    }
}
__device__ __forceinline__ uint32_t bytes_f16(uint32_t x, int sel) { return add_f16(__byte_perm(x ^ 0x80808080u, 0x64646464u, sel), AQ_F16_128); }
__device__ __forceinline__ uint32_t nibble_bf16(uint32_t x, int n) { return add_bf16(((x >> (4 * n)) & 0x000f000fu) | 0x43004300u, 0xc308c308u); }      // -136
__device__ __forceinline__ uint32_t byte_pair_bf16(uint32_t a, uint32_t b, int n)      // byte n of two words (codes plus 128)
{
    const float x = __uint_as_float(__byte_perm(a, 0x4b000000u, 0x7440 + n)), y = __uint_as_float(__byte_perm(b, 0x4b000000u, 0x7440 + n));
    return pack_bf16(x - 8388736.f, y - 8388736.f);
}
// Bytes n and n + 1 (n even) of two words as pairs.
__device__ __forceinline__ void byte_pairs(uint32_t &lo, uint32_t &hi, uint32_t a, uint32_t b, int n)
{
    const uint32_t x = __byte_perm(a, b, n == 0 ? 0x5410 : 0x7632);
    lo = x & 0x00ff00ffu;
    hi = __byte_perm(x, 0u, 0x4341);
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

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

// A warp's way through its part of the keys: which it is, and the ring of stages that it copies them through.
template <int BITS, int D>
struct QuantWalk {
    typedef QuantStage<BITS, D> Stage;
    typedef QuantRow<BITS, D> Row;
    static constexpr int ST = Stage::STAGES, KEYS = Stage::KEYS, RB = Row::BYTES, CH = RB / 16, LR = 32 / CH, SB = Row::SCALE_BYTES, NEXT = AF_WARPS * KEYS;
    const QuantDev &c;
    KeyRange kr;
    int v0, v1;                            // the part: keys v0 .. v1 - 1 of the walk
    int wa, wb;                            // keys wa .. wb - 1 are seen by every row of the tile
    uint32_t ring, own_chunk, own_scale;
    // This warp's stages begin at keys v0 + warp KEYS and every fourth stage from there.  The next one to be fetched has its rows at kp,
    // vp (row lr of it) and scales at ksp, vsp (row `lane`) if it lies whole behind the sinks; where it does not, each row's place is worked out.
    const uint8_t *kp, *vp, *ksp, *vsp;
    int lane, lr, lc;
    bool dense;                            // rows are neighbours in memory: constant steps

    __device__ __forceinline__ QuantWalk(const AttendDev &p, const QuantDev &c, unsigned char *sm, int b, int h, int len, int ql, int i0, int i1, int part, int parts)
        : c(c), kr{0, 0, 0}
    {
        const int warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        lc = lane % CH;
        lr = lane / CH;
        const int t0 = len - ql + i0, t1 = len - ql + i1;
        if (i0 <= i1) kr = attend_range(p, t0, t1, len);
        const int n = kr.count(), per = ((n + 63) / 64 + parts - 1) / parts * 64;
        v0 = min((long long)part * per, (long long)n);
        v1 = min(v0 + per, n);
        wa = 0;
        wb = v1;
        if (p.n_q > 1) {
            wb = min(v1, kr.s + max(0, t0 + 1 - kr.lo));
            if (p.window && t1 - p.window + 1 > kr.lo) wa = kr.s + t1 - p.window + 1 - kr.lo;
        }
        ring = (uint32_t)__cvta_generic_to_shared(sm) + warp * ST * Stage::BYTES;
        own_chunk = ring + chunk_at<RB>(lr, lc);
        own_scale = ring + 2 * Stage::CODES + lane * SB;
        const long long j0 = (long long)v0 + warp * KEYS - kr.s + kr.lo;
        kp = c.k + b * c.ks[0] + h * c.ks[1] + (j0 + lr) * c.ks[2] + lc * 16;
        vp = c.v + b * c.vs[0] + h * c.vs[1] + (j0 + lr) * c.vs[2] + lc * 16;
        ksp = c.k_scale + b * c.kss[0] + h * c.kss[1] + (j0 + lane) * c.kss[2];
        vsp = c.v_scale + b * c.vss[0] + h * c.vss[1] + (j0 + lane) * c.vss[2];
        dense = c.ks[2] == RB && c.vs[2] == RB;
#pragma unroll
        for (int s = 0; s < ST - 1; ++s) fetch(v0 + (warp + s * AF_WARPS) * KEYS, s);
    }
    __device__ __forceinline__ int first() const { return v0 + (int)(threadIdx.x >> 5) * KEYS; }
    __device__ __forceinline__ bool whole(int va) const { return va >= wa && va + KEYS <= wb; }

    __device__ __forceinline__ void fetch(int va, int slot)
    {
        const uint32_t off = slot * Stage::BYTES;
        if (va >= kr.s && va + KEYS <= v1) {
            // (rows LR apart stand alike, but that at 128 bytes every second one has its chunks' halves exchanged)
            const uint32_t at[2] = {own_chunk + off, (RB == 128 ? own_chunk ^ 64u : own_chunk) + off};
            if (dense) {
#pragma unroll
                for (int i = 0; i < KEYS / LR; ++i) {
                    cp_async_all<16>(at[i & 1] + i * LR * RB, kp + i * LR * RB);
                    cp_async_all<16>(at[i & 1] + i * LR * RB + Stage::CODES, vp + i * LR * RB);
                }
            } else {
#pragma unroll
                for (int i = 0; i < KEYS / LR; ++i) {
                    cp_async_all<16>(at[i & 1] + i * LR * RB, kp + i * LR * c.ks[2]);
                    cp_async_all<16>(at[i & 1] + i * LR * RB + Stage::CODES, vp + i * LR * c.vs[2]);
                }
            }
            if (KEYS == 32 || lane < KEYS) {
                cp_async_all<SB>(own_scale + off, ksp);
                cp_async_all<SB>(own_scale + off + Stage::SCALES, vsp);
            }
        } else if (va < v1) {
            const int at_va = va - kr.s + kr.lo;
#pragma unroll 1
            for (int i = 0; i < KEYS / LR; ++i) {
                const int r = lr + i * LR, v = va + r;
                const bool real = v < v1;                 // (behind the part: zeros, whatever the cache holds there)
                const long long step = kr.key(real ? v : v0) - (at_va + lr);
                const uint32_t at = ring + off + chunk_at<RB>(r, lc);
                cp_async16(at, kp + step * c.ks[2], real);
                cp_async16(at + Stage::CODES, vp + step * c.vs[2], real);
            }
            if (lane < KEYS) {
                const int v = va + lane;
                const bool real = v < v1;
                const long long step = kr.key(real ? v : v0) - (at_va + lane);
                cp_async_small<SB>(own_scale + off, ksp + step * c.kss[2], real);
                cp_async_small<SB>(own_scale + off + Stage::SCALES, vsp + step * c.vss[2], real);
            }
        }
        cp_commit();
        kp += NEXT * c.ks[2];
        vp += NEXT * c.vs[2];
        ksp += NEXT * c.kss[2];
        vsp += NEXT * c.vss[2];
    }
    // Waits for the stage of keys va .., in `slot`, and has the one behind those under way fetched to the slot that was read last.
    __device__ __forceinline__ void next(int va, int slot)
    {
        cp_wait<ST - 2>();
        __syncwarp();
        fetch(va + (ST - 1) * NEXT, slot == 0 ? ST - 1 : slot - 1);
    }
};

// Blocks of a multiprocessor, as registers allow.  (16 x 16 query rows over 8192 keys in 8 bits: 3 blocks 64 us, 2 blocks 72; in 4 bits, where 3 spill,
// 67 and 65, 64 query rows 199 and 185.)
template <typename TIN, int BITS, int D, int NT>
constexpr int AQ_BLOCKS = D == 64 ? (sizeof(TIN) == 4 ? (NT == 2 ? 3 : 2) : NT == 2 ? 4 : 3) : sizeof(TIN) == 2 && NT == 2 && BITS == 8 ? 3 : 2;

// A tile's queries, which all warps of a block read over and over: fragments, what the codes' offsets add up to, factors of the logits.
template <typename TIN, int BITS, int D, int NT>
struct QuantQueries {
    static constexpr int PARTS = sizeof(TIN) == 4 ? 2 : 1, KS = D / 16, GR = QuantRow<BITS, D>::GROUPS;
    uint2 frag[PARTS][NT][KS][32];
    float off[NT][GR][8], c[NT][8];
};

template <typename TIN, int BITS, int D, int NT, bool CLUSTER>
__global__ void __launch_bounds__(AF_NT, (AQ_BLOCKS<TIN, BITS, D, NT>)) k_attend_quant(const __grid_constant__ AttendDev p, const __grid_constant__ QuantDev c)
{
    extern __shared__ __align__(128) unsigned char aq_sm[];
    typedef QuantStage<BITS, D> Stage;
    typedef QuantRow<BITS, D> Row;
    constexpr int KS = D / 16, ROWS = 8 * NT, ST = Stage::STAGES, KEYS = Stage::KEYS, RB = Row::BYTES, SB = Row::SCALE_BYTES, GR = Row::GROUPS, SUB = KEYS / 16;
    constexpr int IL = NT <= 2 ? SUB : 1;                 // runs of sixteen keys worked on side by side
    constexpr int PARTS = sizeof(TIN) == 4 ? 2 : 1;       // of a query
    constexpr int WPARTS = sizeof(TIN) == 4 ? 3 : 1;      // of a weight
    constexpr bool EXACT = sizeof(TIN) == 4;              // codes at their full size
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

    const int i0 = tile * ROWS / p.G, i1 = min((min((tile + 1) * ROWS, rows_seq) - 1) / p.G, ql - 1);
    QuantWalk<BITS, D> walk(p, c, aq_sm, b, h, len, ql, i0, i1, part, parts);
    const uint32_t ring = walk.ring;

    // Queries as B fragments: of row 8 nt + lane / 4 a lane holds a quarter of the channels, those of its words of a key.
    auto &qs = *reinterpret_cast<QuantQueries<TIN, BITS, D, NT> *>(aq_sm + AQ_RING<BITS, D>);
    for (int nt = warp; nt < NT; nt += AF_WARPS) {
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
        float sum[GR];
#pragma unroll
        for (int j = 0; j < GR; ++j) sum[j] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            uint2 frag[PARTS];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                // the pair's two channels among the lane's (4 bits: those of u = 1 meet codes sixteen times as large)
                const int a = BITS == 8 ? 4 * k + 2 * u : 2 * k + u, a2 = BITS == 8 ? a + 1 : a + D / 8;
                const float f = BITS == 4 && u == 1 ? up * 0.0625f : up;
                float y = q[a] * f, z = q[a2] * f;
#pragma unroll
                for (int part_q = 0; part_q < PARTS; ++part_q) {
                    const __half2 v = __floats2half2_rn(y, z);
                    (u ? frag[part_q].y : frag[part_q].x) = *reinterpret_cast<const uint32_t *>(&v);
                    y -= __low2float(v);
                    z -= __high2float(v);
                    sum[BITS == 8 ? 0 : k >> 1] += (__low2float(v) + __high2float(v)) * (BITS == 4 && u == 1 ? 16.f : 1.f);
                }
            }
#pragma unroll
            for (int part_q = 0; part_q < PARTS; ++part_q) qs.frag[part_q][nt][k][lane] = frag[part_q];
        }
#pragma unroll
        for (int j = 0; j < GR; ++j) {
            sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 1);
            sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 2);
            qs.off[nt][j][g8] = sum[j] * (BITS == 4 ? -0x1p-21f : -0x1p-17f);       // -8, -128 times 2^-24
        }
        qs.c[nt][g8] = p.c * (EXACT ? 1.f : 0x1p24f) * down;
    }
    __syncthreads();
    float row_c[NT][2];                                   // what makes logits (log2) of a product's rows 8 nt + 2 (lane mod 4) + e
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) row_c[nt][e] = qs.c[nt][2 * t4 + e];

    float o[NT][KS][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) { m[nt][e] = AQ_NONE; l[nt][e] = 0.f; }
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][k][e] = 0.f;
    }
    // Row r of a 16-key product stands for key  r / 2 + 4 (r mod 2)  of its half of eight: a lane then reads four neighbouring keys' values.
    const int key_s = (g8 >> 1) + 4 * (g8 & 1);
    // What this lane reads of sixteen keys: of K words of keys key_s and key_s + 8, of V words of keys lane mod 4 + 4 i, the second half of
    // eight keys 8 rows behind the first in both; scales of keys key_s and key_s + 8.
    constexpr int W = RB / 32;                            // words of V
    const uint32_t k_at = ring + (RB == 32 ? chunk_at<RB>(key_s, t4 >> 1) + (t4 & 1) * 8 : chunk_at<RB>(key_s, t4));
    uint32_t v_at[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        v_at[i] = ring + Stage::CODES + (W == 4 ? chunk_at<RB>(t4 + 4 * i, g8) : W == 2 ? chunk_at<RB>(t4 + 4 * i, g8 >> 1) + (g8 & 1) * 8 : chunk_at<RB>(t4 + 4 * i, g8 >> 2) + (g8 & 3) * 4);
    const uint32_t s_at = ring + 2 * Stage::CODES + key_s * SB;
    int slot = 0;
    for (int va = walk.first(); va < walk.v1; va += AF_WARPS * KEYS) {
        walk.next(va, slot);
        const uint32_t off = slot * Stage::BYTES, kd = k_at + off, vd0 = v_at[0] + off, vd1 = v_at[1] + off, sd = s_at + off;
        float s[SUB][NT][4];
        // ---- logits (products that wait for one another are kept apart by those of other rows and of the other sixteen keys) ----
#pragma unroll
        for (int s0 = 0; s0 < SUB; s0 += IL) {
        if constexpr (BITS == 4) {
            constexpr int KW = D / 32;                    // words of a lane
            uint32_t w0[IL][KW], w1[IL][KW], f0[IL][GR / 2], f1[IL][GR / 2];
#pragma unroll
            for (int sub = 0; sub < IL; ++sub) {
                lds(w0[sub], kd + (s0 + sub) * 16 * RB);
                lds(w1[sub], kd + ((s0 + sub) * 16 + 8) * RB);
                lds(f0[sub], sd + (s0 + sub) * 16 * SB);
                lds(f1[sub], sd + ((s0 + sub) * 16 + 8) * SB);
            }
#pragma unroll
            for (int j = 0; j < GR; ++j) {
                const int sel = j & 1 ? 0x7632 : 0x5410;
                uint32_t n0[IL][4], n1[IL][4];
                float acc[IL][NT][4];
#pragma unroll
                for (int sub = 0; sub < IL; ++sub) {
                    const uint32_t y = __byte_perm(w0[sub][j >> 1], w0[sub][(j >> 1) + KW / 2], sel), z = __byte_perm(w1[sub][j >> 1], w1[sub][(j >> 1) + KW / 2], sel);
                    if constexpr (EXACT) {
                        nibbles_f16(n0[sub], y);
                        nibbles_f16(n1[sub], z);
                    } else {
                        nibbles(n0[sub], y);
                        nibbles(n1[sub], z);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int part_q = PARTS - 1; part_q >= 0; --part_q)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint2 qf = qs.frag[part_q][nt][2 * j + i][lane];
#pragma unroll
                            for (int sub = 0; sub < IL; ++sub) {
                                const uint32_t a[4] = {n0[sub][2 * i], n1[sub][2 * i], n0[sub][2 * i + 1], n1[sub][2 * i + 1]};
                                if (i == 0 && part_q == PARTS - 1) mma_f16_first(acc[sub][nt], a, qf.x, qf.y);
                                else mma_f16(acc[sub][nt], a, qf.x, qf.y);
                            }
                        }
#pragma unroll
                for (int sub = 0; sub < IL; ++sub) {
                    const float k0 = j & 1 ? bf16_hi(f0[sub][j >> 1]) : bf16_lo(f0[sub][j >> 1]), k1 = j & 1 ? bf16_hi(f1[sub][j >> 1]) : bf16_lo(f1[sub][j >> 1]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float f = e < 2 ? k0 : k1, y = EXACT ? acc[sub][nt][e] : acc[sub][nt][e] + qs.off[nt][j][2 * t4 + (e & 1)];
                            s[s0 + sub][nt][e] = j == 0 ? y * f : fmaf(y, f, s[s0 + sub][nt][e]);
                        }
                }
            }
        } else {
            float acc[IL][NT][2][4];
#pragma unroll
            for (int half = 0; half < KS / 4; ++half) {
                uint32_t w0[IL][4], w1[IL][4];
#pragma unroll
                for (int sub = 0; sub < IL; ++sub) {
                    lds(w0[sub], (half ? kd ^ 64u : kd) + (s0 + sub) * 16 * RB);       // (rows of 128 bytes: chunks t and t + 4)
                    lds(w1[sub], (half ? kd ^ 64u : kd) + ((s0 + sub) * 16 + 8) * RB);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int sub = 0; sub < IL; ++sub) {
                        const int k = 4 * half + i;
                        uint32_t a[4];
                        if constexpr (EXACT) {
                            a[0] = bytes_f16(w0[sub][i], 0x4140);
                            a[1] = bytes_f16(w1[sub][i], 0x4140);
                            a[2] = bytes_f16(w0[sub][i], 0x4342);
                            a[3] = bytes_f16(w1[sub][i], 0x4342);
                        } else {
                            const uint32_t x = w0[sub][i] ^ 0x80808080u, y = w1[sub][i] ^ 0x80808080u;
                            a[0] = __byte_perm(x, 0u, 0x4140);
                            a[1] = __byte_perm(y, 0u, 0x4140);
                            a[2] = __byte_perm(x, 0u, 0x4342);
                            a[3] = __byte_perm(y, 0u, 0x4342);
                        }
#pragma unroll
                        for (int part_q = PARTS - 1; part_q >= 0; --part_q)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                const uint2 qf = qs.frag[part_q][nt][k][lane];
                                if (k < 2 && part_q == PARTS - 1) mma_f16_first(acc[sub][nt][k], a, qf.x, qf.y);
                                else mma_f16(acc[sub][nt][k & 1], a, qf.x, qf.y);
                            }
                    }
            }
#pragma unroll
            for (int sub = 0; sub < IL; ++sub) {
                const float k0 = __uint_as_float(lds1(sd + (s0 + sub) * 16 * SB)), k1 = __uint_as_float(lds1(sd + ((s0 + sub) * 16 + 8) * SB));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[s0 + sub][nt][e] = (acc[sub][nt][0][e] + acc[sub][nt][1][e] + (EXACT ? 0.f : qs.off[nt][0][2 * t4 + (e & 1)])) * (e < 2 ? k0 : k1);
            }
        }
        }
        // ---- weights: s[sub][nt][2 u + e] is key 8 u + key_s of sixteen, row 8 nt + 2 (lane mod 4) + e ----
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[sub][nt][e] *= row_c[nt][e & 1];
        if (!walk.whole(va)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int t = len - ql + (tile * ROWS + nt * 8 + 2 * t4 + e) / p.G;         // (of rows that are none: anything)
#pragma unroll
                    for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int v = va + 16 * sub + key_s + 8 * u;
                            if (v >= walk.v1 || !attend_sees(p, t, walk.kr.key(v))) s[sub][nt][2 * u + e] = -INFINITY;
                        }
                }
        }
        float over = -INFINITY;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = fmaxf(s[0][nt][e], s[0][nt][2 + e]);
#pragma unroll
                for (int sub = 1; sub < SUB; ++sub) top = fmaxf(top, fmaxf(s[sub][nt][e], s[sub][nt][2 + e]));
                over = fmaxf(over, top - m[nt][e]);
            }
        if (__any_sync(0xffffffffu, over > AF_RAISE)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float mx = s[0][nt][e];
#pragma unroll
                    for (int sub = 0; sub < SUB; ++sub) mx = fmaxf(mx, fmaxf(s[sub][nt][e], s[sub][nt][2 + e]));
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                    mx = fmaxf(mx, m[nt][e]);
                    const float f = ex2(m[nt][e] - mx);
                    m[nt][e] = mx;
                    l[nt][e] *= f;
#pragma unroll
                    for (int k = 0; k < KS; ++k) { o[nt][k][e] *= f; o[nt][k][2 + e] *= f; }
                }
        }
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[sub][nt][e] = aq_weight<TIN>(s[sub][nt][e], m[nt][e & 1]);
                    l[nt][e & 1] += s[sub][nt][e];
                }
        // ---- values ----
        if constexpr (BITS == 4) {
#pragma unroll
            for (int s0 = 0; s0 < SUB; s0 += IL) {
            uint32_t w[IL][4][W], f0[IL][GR / 2], f1[IL][GR / 2];            // of keys lane mod 4 + 4 i
#pragma unroll
            for (int sub = 0; sub < IL; ++sub) {
#pragma unroll
                for (int i = 0; i < 4; ++i) lds(w[sub][i], (i & 1 ? vd1 : vd0) + ((s0 + sub) * 16 + (i & 2) * 4) * RB);
                lds(f0[sub], sd + Stage::SCALES + (s0 + sub) * 16 * SB);
                lds(f1[sub], sd + Stage::SCALES + ((s0 + sub) * 16 + 8) * SB);
            }
#pragma unroll
            for (int j = 0; j < GR; ++j) {
                const int sel = j & 1 ? 0x7632 : 0x5410;
                uint32_t pf[IL][NT][WPARTS][2], ab[IL][4], cd[IL][4];
#pragma unroll
                for (int sub = 0; sub < IL; ++sub) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const uint32_t fw = u ? f1[sub][j >> 1] : f0[sub][j >> 1];
                            const float f = j & 1 ? bf16_hi(fw) : bf16_lo(fw);
                            uint32_t pw[WPARTS];
                            split_weights<WPARTS>(pw, s[s0 + sub][nt][2 * u] * f, s[s0 + sub][nt][2 * u + 1] * f);
#pragma unroll
                            for (int q = 0; q < WPARTS; ++q) pf[sub][nt][q][u] = transpose8x8(pw[q]);
                        }
                    const uint32_t y = __byte_perm(w[sub][0][j >> 1], w[sub][1][j >> 1], sel), z = __byte_perm(w[sub][2][j >> 1], w[sub][3][j >> 1], sel);
                    if constexpr (!EXACT) {
                        nibbles(ab[sub], y);
                        nibbles(cd[sub], z);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        ab[sub][i] = EXACT ? nibble_bf16(y, i) : add_bf16(ab[sub][i], i & 1 ? AQ_MINUS_128 : AQ_MINUS_8);
                        cd[sub][i] = EXACT ? nibble_bf16(z, i) : add_bf16(cd[sub][i], i & 1 ? AQ_MINUS_128 : AQ_MINUS_8);
                    }
                }
#pragma unroll
                for (int sub = 0; sub < IL; ++sub)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t a[4] = {ab[sub][2 * i], ab[sub][2 * i + 1], cd[sub][2 * i], cd[sub][2 * i + 1]};
                            mma_weights<EXACT, WPARTS>(o[nt][2 * j + i], a, pf[sub][nt]);
                        }
            }
            }
        } else {
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) {
                uint32_t w[4][W], pf[NT][WPARTS][2];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lds(w[i], (i & 1 ? vd1 : vd0) + (sub * 16 + (i & 2) * 4) * RB);
#pragma unroll
                    for (int q = 0; q < W; ++q) w[i][q] ^= 0x80808080u;
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float f = __uint_as_float(lds1(sd + Stage::SCALES + (sub * 16 + 8 * u) * SB));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        uint32_t pw[WPARTS];
                        split_weights<WPARTS>(pw, s[sub][nt][2 * u] * f, s[sub][nt][2 * u + 1] * f);
#pragma unroll
                        for (int q = 0; q < WPARTS; ++q) pf[nt][q][u] = transpose8x8(pw[q]);
                    }
                }
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    uint32_t a[4];
                    if constexpr (EXACT) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[e] = byte_pair_bf16(w[e & 2][i >> 1], w[(e & 2) + 1][i >> 1], 2 * (i & 1) + (e & 1));
                    } else {
                        byte_pairs(a[0], a[1], w[0][i >> 1], w[1][i >> 1], 2 * (i & 1));
                        byte_pairs(a[2], a[3], w[2][i >> 1], w[3][i >> 1], 2 * (i & 1));
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[e] = add_bf16(a[e], AQ_MINUS_128);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_weights<EXACT, WPARTS>(o[nt][i], a, pf[nt]);
                }
            }
        }
        slot = slot + 1 == ST ? 0 : slot + 1;
    }
    cp_wait<0>();
    __syncthreads();

    // the warps' results: O as [warp][row][D + 4], then references and sums; tile k of O holds channels (lane / 4) D / 8 + 2 k, + 1
    constexpr int LD = D + 4;
    constexpr float U = AQ_VALUE<TIN>, U2 = BITS == 4 && !EXACT ? U * 0.0625f : U;         // (4 bits: every second pair is sixteenfold)
    float *osm = reinterpret_cast<float *>(aq_sm), *ml = osm + AF_WARPS * ROWS * LD;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float z = l[nt][e];
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) z += __shfl_xor_sync(0xffffffffu, z, w);
            const int row = 8 * nt + 2 * t4 + e;
            if (lane < 4) { ml[(warp * ROWS + row) * 2] = m[nt][e]; ml[(warp * ROWS + row) * 2 + 1] = z * AQ_SUM<TIN>; }
#pragma unroll
            for (int k = 0; k < KS; k += 2)
                *reinterpret_cast<float4 *>(&osm[(warp * ROWS + row) * LD + g8 * (D / 8) + 2 * k]) = make_float4(o[nt][k][e] * U, o[nt][k][2 + e] * U2, o[nt][k + 1][e] * U, o[nt][k + 1][2 + e] * U2);
        }
    __syncthreads();
    few_finish<TIN, D, ROWS, false, CLUSTER>(p, osm, ml, tile, part, parts, rows_seq, rows_seq, h, b, len, ql, walk.kr, walk.v0, walk.v1, AQ_LSE<TIN>);
}

}  // namespace obf
