// Attention of many query rows per KV head on the tensor cores (bf16): prompts, chunks of queries, a batch over a shared prefix.
//
// A block (one per multiprocessor, persistent) works on items: two tiles of up to 128 query rows of a KV head and a part of the
// keys that they see.  A tile is `ti` queries x the G heads of the group (so its rows see nearly the same keys and a window
// wastes little), over a shared prefix, where all rows see the same, also `nb` sequences: as many of either as make the fewest tiles.  Keys come in tiles of 128: the sinks first, padded with
// zeros to 16, 32, 48 or 64 rows (more of them: to whole tiles), the window's range behind them in the same tile.
//   warp 2, a thread    works out the items (ahead of the others, who read them from shared memory); Q, K and V tiles by TMA
//                       (128-byte swizzle) into a ring of K and V slots
//   warps 0, 1          products of the first and the second query tile: S = Q K^T into tensor memory, O += P V with P from
//                       tensor memory; those of one tile run while the softmax of the other does
//   warps 4-11, 12-19   softmax of the first and the second query tile, two threads per row with 64 keys each (one warp alone on a
//                       scheduler leaves the special-function unit idle between its instructions), weights to bf16 over the logits' columns
//                       (a product takes both operands in one 16-bit type, and the values are bf16; off by at most 2^-8 of a weight, a bf16 output
//                       by 2.3e-3 of its norm where its own rounding alone makes 1.7e-3), their fp32 sum; after the last tile O / sum to memory
//
// Softmax: fp32 and bf16 have the same exponents, so a row's reference need not be its maximum, only near enough for no weight
// to leave fp32's range.  It starts as zero, and the logits are read once, without a search for their maximum before.  Only when
// 64 weights add up to more than 2^32, or those of a row's first tile to less than 2^-40 (logits beyond some 18 to 22, or -28; rows that
// see nothing of that tile), is the tile done again against the rows' maxima, O and the sums rescaled - in place: the products
// before have completed, since they were issued before the logits that the thread has waited for.  n keys' weights add up to less
// than 2^26 (n + 128), so values of up to 2^90, and of up to 2^100 / n, overflow nothing.
// Tensor memory: S (P) and O of the two tiles, 512 columns.  Every wait is bounded.
//
// Rows of V past the last key may hold anything, and 0 * NaN is not 0: the product over a short tile runs over its keys rounded
// up to 16, and the softmax warps clear the rows in between.
//
// Bound by the exponentials (16 per cycle and multiprocessor: 1024 cycles a tile of 128 x 128) and the two products (512 cycles
// each) alike, and by the chain from one to the other: a pair of tiles takes 2900 to 3200 cycles, not 2048.  Prompt of 8192, 32
// heads over 8, 128 channels: causal 552 us (997 TFLOP/s, 60 % of the measured burst rate), with a window of 1024 and 4 sinks 161
// us (805; 175 in long runs, at the power limit).
#pragma once

#include "attend_common.cuh"
#include "tc_common.cuh"

namespace obf {

constexpr int AT_TILE = 128;
constexpr int AT_THREADS = 640;
// A thread's 64 weights of a tile may add up to 2^32 (those of an item's first tile have to reach 2^-40).  More than that takes a logit
// of more than 26 above the reference (log2), so a tile turned down for it raises the reference, whose margin of 25 leaves room for the
// rounding of the sum.
constexpr float AT_FUSED_MAX = 4096.f;
constexpr float AT_RAISE = 25.f, AT_WEIGHT_MAX = 4294967296.f, AT_WEIGHT_MIN = 9.094947017729282e-13f;     // 2^32, 2^-40

template <int D>
struct AttendTcShape {
    static constexpr int SLOT_BYTES = AT_TILE * D * 2;                    // a tile of Q, K or V
    static constexpr int SLOTS = D == 128 ? 5 : 8;
    static constexpr int SMEM_BYTES = (2 + SLOTS) * SLOT_BYTES;           // beside what the kernel declares, and alignment to 1024
};

// Tensor maps and tile shape of the kernel.
struct AttendTcMaps {
    CUtensorMap q, k, v;
    CUtensorMap head[2], rest[2];                                         // K and V: the sinks, and what the sinks leave of a tile
    int32_t ti, nb;                                                       // queries and sequences of a tile of rows
    int32_t head_rows;                                                    // rows that the sinks take: at most 64, or whole tiles
};

// What every role of a block knows about an item.
template <bool PREFIX>
struct AttendTcItem {
    int h, b, part;                  // KV head, sequence (of own keys), part of the keys
    int ti, nb;                      // queries and sequences of a tile
    int fi[2], fb[2];                // first query and sequence of the tiles
    int head, lo, hi;                // keys of the pair: the sinks in `head` rows (zeros behind them), then lo .. hi - 1
    int jb, je;                      // the part's tiles
    // per tile of rows: some row sees tile j of the keys when j < sk or ja <= j < jz, every row sees all of it when fa <= j < fz
    int sk[2], ja[2], jz[2], fa[2], fz[2];
    bool valid[2];
    int t;                           // position of a sequence's first query
    int ql;

    __device__ __forceinline__ void init(const AttendDev &p, const AttendTcMaps &tm, int item)
    {
        ti = tm.ti;
        nb = tm.nb;
        const int parts = PREFIX ? p.p_slots : p.slots - p.p_slots;
        part = item % parts;
        item /= parts;
        h = item % p.kv_heads;
        item /= p.kv_heads;
        b = head = lo = hi = t = ql = 0;
        if (PREFIX) {
            hi = p.prefix;
            const int groups = (p.batch + nb - 1) / nb;                   // of sequences; tiles go through them first
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int tile = 2 * item + x;
                fi[x] = tile / groups * ti;
                fb[x] = tile % groups * nb;
                valid[x] = fi[x] < p.n_q;
                sk[x] = ja[x] = fa[x] = 0;
                jz[x] = valid[x] ? (hi + AT_TILE - 1) / AT_TILE : 0;
                fz[x] = hi / AT_TILE;
            }
        } else {
            b = item % p.batch;
            item /= p.batch;
            const int pairs = (p.n_q + 2 * ti - 1) / (2 * ti);
            const int i0 = (pairs - 1 - item) * 2 * ti;                   // the longest key ranges first
            fi[0] = i0;
            fi[1] = i0 + ti;
            fb[0] = fb[1] = b;
            const int len = attend_len(p, b);
            ql = attend_q_len(p, b);
            t = len - ql;
            valid[0] = i0 < ql;
            valid[1] = i0 + ti < ql;
            if (valid[0]) {
                const KeyRange r = attend_range(p, t + i0, t + min(i0 + 2 * ti, ql) - 1, len);
                hi = r.hi;
                if (r.lo > p.sinks) {
                    lo = r.lo;
                    head = p.sinks ? tm.head_rows : 0;
                }
                // up to a multiple of 16 keys where there are more, which later queries see
                hi = min(len, hi + (lo - hi - head & 15));
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                sk[x] = ja[x] = jz[x] = fa[x] = fz[x] = 0;
                if (valid[x]) {
                    const int ta = t + i0 + x * ti, tb = t + min(i0 + (x + 1) * ti, ql) - 1;      // positions of its first and last query
                    const KeyRange r = attend_range(p, ta, tb, len);
                    sk[x] = (head + AT_TILE - 1) / AT_TILE;
                    ja[x] = p.sinks > lo ? 0 : (head + r.lo - lo) / AT_TILE;
                    jz[x] = r.hi > lo ? (head + r.hi - lo + AT_TILE - 1) / AT_TILE : 0;
                    fa[x] = max(sk[x], p.window ? max(head + tb - p.window + 1 - lo + AT_TILE - 1, 0) / AT_TILE : 0);
                    fz[x] = max(head + ta + 1 - lo, 0) / AT_TILE;
                }
            }
        }
        const int tiles = (head + hi - lo + AT_TILE - 1) / AT_TILE, per = (tiles + parts - 1) / parts;
        jb = min(part * per, tiles);
        je = min(jb + per, tiles);
    }

    __device__ __forceinline__ int width(int j) const { return min(AT_TILE, head + hi - lo - j * AT_TILE); }
};

// D[tmem] (+)= A[tmem] * B, K = 16 per instruction: A holds two bf16 of a row per column.
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

// One lane of the warp, always the same.  (Told apart like this the compiler knows that a single thread runs what depends on it, and
// keeps the products' operands in uniform registers.)
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(r));
    return r != 0;
}

// tc::mbar_wait by a whole warp, which goes on as one.
__device__ __forceinline__ bool mbar_wait_warp(uint64_t *bar, uint32_t parity, const tc::WaitCtx &w)
{
    if (__all_sync(0xffffffffu, tc::mbar_try(bar, parity))) return true;
    return __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, w));
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}

__device__ __forceinline__ void tmem_ld_wait16(uint32_t (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int c0, int c1, int c2, int c3)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(tc::smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}

// A box of keys or values: rows from `row` on, column block `block` (all of them for boxes that are that wide).
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int row, int block, int head, int seq)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                 ::"r"(dst), "l"(map), "r"(tc::smem_u32(bar)), "r"(0), "r"(row), "r"(block), "r"(head), "r"(seq) : "memory");
}

// 32 bytes to global memory, in two halves where the address is no multiple of 32.
__device__ __forceinline__ void store32(void *dst, const uint32_t (&r)[8], bool wide)
{
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
    } else {
        reinterpret_cast<uint4 *>(dst)[0] = make_uint4(r[0], r[1], r[2], r[3]);
        reinterpret_cast<uint4 *>(dst)[1] = make_uint4(r[4], r[5], r[6], r[7]);
    }
}

// Bits of columns a .. b - 1 of 32.
__device__ __forceinline__ uint32_t column_bits(int a, int b)
{
    a = max(a, 0);
    b = min(b, 32);
    if (a >= b) return 0u;
    return (0xFFFFFFFFu >> (32 - b)) & (0xFFFFFFFFu << a);
}

template <int D, bool PREFIX>
__global__ void __launch_bounds__(AT_THREADS, 1) k_attend_tc(const __grid_constant__ AttendDev p, const __grid_constant__ AttendTcMaps tm, const int items,
                                                           const int first)
{
    constexpr int SLOTS = AttendTcShape<D>::SLOTS, SLOT_BYTES = AttendTcShape<D>::SLOT_BYTES, BLOCK = AT_TILE * 128, NB = D / 64;
    extern __shared__ uint8_t at_smem_raw[];
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(at_smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t *q_sm = base, *ring = base + 2 * SLOT_BYTES;
    __shared__ uint64_t bar_full[SLOTS], bar_empty[SLOTS], bar_q_full, bar_q_empty, bar_drain[2];
    __shared__ uint64_t bar_s[2], bar_p[2], bar_o[2], bar_o_read[2], bar_item[2], bar_item_read[2], bar_turn[2];
    __shared__ AttendTcItem<PREFIX> sm_item[2];
    __shared__ float sm_row[2][2][AT_TILE];               // a row's two threads trade their maxima and sums
    __shared__ uint32_t s_tmem, s_abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    {
        uint32_t given;
        asm("mov.u32 %0, %%dynamic_smem_size;" : "=r"(given));
        if ((uint32_t)(base - at_smem_raw) + AttendTcShape<D>::SMEM_BYTES > given) {      // (the launch and this layout belong together)
            if (tid == 0) atomicOr(p.status, OBF_DEV_INTERNAL);
            return;
        }
    }
    tc::WaitCtx wc{&s_abort, p.status, p.wait_limit_ns};
    if (tid == 0) {
        s_abort = 0u;
        for (int i = 0; i < SLOTS; ++i) { tc::mbar_init(&bar_full[i], 1); tc::mbar_init(&bar_empty[i], 2); }
        tc::mbar_init(&bar_q_full, 1);
        tc::mbar_init(&bar_q_empty, 2);
        for (int x = 0; x < 2; ++x) {
            tc::mbar_init(&bar_s[x], 1);
            tc::mbar_init(&bar_p[x], 8);
            tc::mbar_init(&bar_o[x], 1);
            tc::mbar_init(&bar_o_read[x], 8);
            tc::mbar_init(&bar_item[x], 1);
            tc::mbar_init(&bar_item_read[x], 18);
            tc::mbar_init(&bar_drain[x], 1);
            tc::mbar_init(&bar_turn[x], 1);
        }
        tc::mbar_init_fence();
    }
    if (warp == 0) tc::tmem_alloc(&s_tmem, 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = s_tmem;
    if (first) pdl_wait();                               // (else as in k_attend_few)
    pdl_trigger();
    if (first && blockIdx.x == 0) attend_status(p);

    AttendTcItem<PREFIX> it;
    if (warp == 2) {
        // ---------------- copies ----------------
        if (lane == 0) {
            uint32_t n = 0, nq = 0, ni = 0;
            bool dead = false;
            for (int item = blockIdx.x; item < items && !dead; item += gridDim.x, ++ni) {
                it.init(p, tm, item);
                if (!tc::mbar_wait(&bar_item_read[ni & 1u], ((ni >> 1) & 1u) ^ 1u, wc)) break;
                sm_item[ni & 1u] = it;
                tc::mbar_arrive(&bar_item[ni & 1u]);
                if (it.jb >= it.je) continue;
                for (int j = it.jb; j < it.je && !dead; ++j) {
                    for (int kv = 0; kv < 2; ++kv, ++n) {
                        const uint32_t sl = n % SLOTS;
                        if (!tc::mbar_wait(&bar_empty[sl], ((n / SLOTS) & 1u) ^ 1u, wc)) { dead = true; break; }
                        if (p.debug_drop_load && n == 1u) continue;                       // the first values never come
                        tc::mbar_expect_tx(&bar_full[sl], SLOT_BYTES);
                        const uint32_t dst = tc::smem_u32(ring + sl * SLOT_BYTES);
                        const int b = PREFIX ? 0 : it.b, j0 = j * AT_TILE;
                        if (!PREFIX && j0 < it.head && it.head < AT_TILE) {
                            for (int c = 0; c < NB; ++c) {
                                tma_load_5d(dst + c * BLOCK, &tm.head[kv], &bar_full[sl], 0, c, it.h, b);
                                tma_load_5d(dst + c * BLOCK + it.head * 128, &tm.rest[kv], &bar_full[sl], it.lo, c, it.h, b);
                            }
                        } else if (!PREFIX && j0 < it.head) {
                            tma_load_5d(dst, &tm.head[kv], &bar_full[sl], j0, 0, it.h, b);
                        } else {
                            tma_load_5d(dst, kv ? &tm.v : &tm.k, &bar_full[sl], it.lo + j0 - it.head, 0, it.h, b);
                        }
                    }
                    if (j > it.jb || dead) continue;
                    // the queries behind the first tile of keys, which need not wait until the last item's are done with
                    if (!tc::mbar_wait(&bar_q_empty, (nq & 1u) ^ 1u, wc)) { dead = true; break; }
                    const int rows = p.G * it.ti * it.nb, loads = (it.valid[0] ? NB : 0) + (it.valid[1] ? NB : 0);
                    tc::mbar_expect_tx(&bar_q_full, (uint32_t)(loads * rows * 128));
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (it.valid[x])
                            for (int c = 0; c < NB; ++c)
                                tma_load_4d(tc::smem_u32(q_sm + x * SLOT_BYTES + c * BLOCK), &tm.q, &bar_q_full, 64 * c, it.h * p.G, it.fi[x], it.fb[x]);
                    ++nq;
                }
            }
            // nothing that this thread started may be in flight when the block exits
            for (uint32_t j = n > (uint32_t)SLOTS ? n - SLOTS : 0u; j < n; ++j) tc::mbar_drain(&bar_full[j % SLOTS], (j / SLOTS) & 1u, wc);
            if (nq) tc::mbar_drain(&bar_q_full, (nq - 1) & 1u, wc);
        }
    } else if (warp < 2) {
        // ---------------- products ----------------
        const int x = warp_uniform(warp);
        const uint32_t tm_u = warp_uniform((int)tmem), q_u = warp_uniform((int)tc::smem_u32(q_sm)), ring_u = warp_uniform((int)tc::smem_u32(ring));
        const uint32_t s_t = tm_u + 128 * x, o_t = tm_u + 256 + 128 * x;
        const uint64_t qd = tc::smem_desc_sw128(q_u + x * SLOT_BYTES, 16, 1024);
        constexpr uint32_t idesc_o = tc::idesc_bf16(128, D, 0, 1);
        uint32_t n = 0, nq = 0, ni = 0, ns = 0, no = 0, nt = 0;
        bool dead = false;
        for (int item = blockIdx.x; item < items && !dead; item += gridDim.x, ++ni) {
            if (!mbar_wait_warp(&bar_item[ni & 1u], (ni >> 1) & 1u, wc)) break;
            const AttendTcItem<PREFIX> &im = sm_item[ni & 1u];
            it.jb = warp_uniform(im.jb);
            it.je = warp_uniform(im.je);
            it.head = warp_uniform(im.head);
            it.lo = warp_uniform(im.lo);
            it.hi = warp_uniform(im.hi);
            const int sk = warp_uniform(im.sk[x]), ja = warp_uniform(im.ja[x]), jz = warp_uniform(im.jz[x]);
            if (elect_one()) tc::mbar_arrive(&bar_item_read[ni & 1u]);
            __syncwarp();
            if (it.jb >= it.je) continue;
            if (!mbar_wait_warp(&bar_q_full, nq & 1u, wc)) break;
            ++nq;
            bool pending = false, started = false;
            int w16_prev = 0;
            // ring positions: K of tile j at n + 2 (j - jb), V behind it
            for (int j = it.jb; j <= it.je; ++j) {
                int w16 = 0;
                const uint32_t nk = n + 2 * (j - it.jb), nv = nk - 1, slot_k = nk % SLOTS, slot_v = nv % SLOTS;
                if (j > it.jb) {
                    if (!mbar_wait_warp(&bar_full[slot_v], (nv / SLOTS) & 1u, wc)) { dead = true; break; }
                    if (pending && !started && !mbar_wait_warp(&bar_o_read[x], (no & 1u) ^ 1u, wc)) { dead = true; break; }
                }
                if (j < it.je && !mbar_wait_warp(&bar_full[slot_k], (nk / SLOTS) & 1u, wc)) { dead = true; break; }
                if (pending && !mbar_wait_warp(&bar_p[x], (ns - 1) & 1u, wc)) { dead = true; break; }
                // The two warps take turns: left alone they fall into step, both tiles in their softmax, then both in their products.
                if (!mbar_wait_warp(&bar_turn[x], (nt & 1u) ^ (uint32_t)(x ^ 1), wc)) { dead = true; break; }
                ++nt;
                tc::tc_fence_after();
                const bool was = pending;
                pending = j < it.je && (j < sk || (j >= ja && j < jz));
                if (pending) w16 = (it.width(j) + 15) & ~15;
                if (elect_one()) {
                    if (was) {
                        // 16 keys of V on: 2048 bytes, 128 in the descriptor; their weights: 8 columns (those of the second 64 keys
                        // begin where their logits did, so that a warp's stores touch its own logits alone)
                        const uint64_t vd = tc::smem_desc_sw128(ring_u + slot_v * SLOT_BYTES, BLOCK, 1024);
                        if (w16_prev == AT_TILE) {
#pragma unroll
                            for (int k = 0; k < AT_TILE / 16; ++k) umma_ts(o_t, s_t + 8 * k + (k & 4) * 8, vd + 128 * k, idesc_o, (started || k > 0) ? 1u : 0u);
                        } else {
                            for (int k = 0; k < w16_prev / 16; ++k) umma_ts(o_t, s_t + 8 * k + (k & 4) * 8, vd + 128 * k, idesc_o, (started || k > 0) ? 1u : 0u);
                        }
                        tc::umma_commit(&bar_empty[slot_v]);
                    } else if (j > it.jb) {
                        tc::mbar_arrive(&bar_empty[slot_v]);
                    }
                    if (pending) {
                        const uint64_t kd = tc::smem_desc_sw128(ring_u + slot_k * SLOT_BYTES, 16, 1024);
                        const uint32_t idesc_s = tc::idesc_bf16(128, 0, 0, 0) | ((uint32_t)(w16 >> 3) << 17);
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            // 16 channels on: 32 bytes, every 64 the next column block; descriptors count 16 bytes
                            const uint64_t off = ((k >> 2) * BLOCK + (k & 3) * 32) / 16;
                            tc::umma_bf16(s_t, qd + off, kd + off, idesc_s, k > 0);
                        }
                        tc::umma_commit(&bar_s[x]);
                        tc::umma_commit(&bar_empty[slot_k]);
                    } else if (j < it.je) {
                        tc::mbar_arrive(&bar_empty[slot_k]);
                    }
                    tc::mbar_arrive(&bar_turn[x ^ 1]);
                    if (j == it.je - 1) tc::umma_commit(&bar_q_empty);
                    if (j == it.je && (started || was)) tc::umma_commit(&bar_o[x]);
                }
                started = started || was;
                ns += pending ? 1 : 0;
                w16_prev = w16;
                __syncwarp();
            }
            n += 2 * (it.je - it.jb);
            no += started ? 1 : 0;
        }
        // no product may be in flight when the block exits
        if (elect_one()) {
            tc::umma_commit(&bar_drain[x]);
            tc::mbar_drain(&bar_drain[x], 0, wc);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ---------------- softmax ----------------
        const int sw = warp - 4, x = sw >> 3, half = (sw >> 2) & 1, quarter = warp & 3, row = quarter * 32 + lane, col0 = half * 64;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16, s_t = tmem + 128 * x + lanes, o_t = tmem + 256 + 128 * x + lanes;
        const f32x2 c2 = pk(p.c, p.c);
        // the row's head of the group, and its query and sequence from the tile's first ones on
        const int row_g = row % p.G, row_b = row / p.G / tm.ti, row_i = row / p.G - row_b * tm.ti;
        // Whether the condition holds for some thread of the two warps that share rows.  Both come here the same number of times,
        // after a wait that ran out too, so that they leave together.
        auto any = [&](bool c) {
            uint32_t r;
            tc::tc_fence_before();
            __syncwarp();
            asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %2, 0;\n barrier.cta.red.or.pred.aligned q, %1, 64, p;\n selp.u32 %0, 1, 0, q;\n}"
                         : "=r"(r) : "r"(1 + 4 * x + quarter), "r"((int)c) : "memory");
            tc::tc_fence_after();
            return r != 0;
        };
        uint32_t n = 0, ni = 0, ns = 0, no = 0;
        bool dead = false;
        const bool wide = (((reinterpret_cast<uintptr_t>(p.out) | (uintptr_t)(p.os[0] | p.os[1] | p.os[2]) * 2) & 31u) == 0);
        for (int item = blockIdx.x; item < items && !dead; item += gridDim.x, ++ni) {
            if (any(!tc::mbar_wait(&bar_item[ni & 1u], (ni >> 1) & 1u, wc))) break;
            // (what only the beginning and the end of an item need is read from shared memory both times: registers are short)
            const AttendTcItem<PREFIX> &im = sm_item[ni & 1u];
            const int jb = im.jb, je = im.je, sk = im.sk[x], ja = im.ja[x], jz = im.jz[x], fa = im.fa[x], fz = im.fz[x];
            it.head = im.head;
            it.lo = im.lo;
            it.hi = im.hi;
            bool real = im.valid[x] && row_b < im.nb;
            {
                const int i = im.fi[x] + row_i, b = im.fb[x] + row_b;
                real = real && b < p.batch && i < (PREFIX ? attend_q_len(p, min(b, p.batch - 1)) : im.ql);
            }
            const int t = PREFIX || !real ? 0 : im.t + im.fi[x] + row_i;
            float m = 0.f;
            f32x2 l2 = 0ull;
            bool started = false, known = true;           // known: all rows have references
            for (int j = jb; j < je; ++j) {
                if (!(j < sk || (j >= ja && j < jz))) continue;
                const bool late = !tc::mbar_wait(&bar_s[x], ns & 1u, wc);
                ++ns;
                __syncwarp();
                tc::tc_fence_after();
                const int width = it.width(j);
                // of 32 columns from col0 + 32 c on, those that the row sees
                auto seen = [&](int c) {
                    uint32_t bits = column_bits(0, width - col0 - 32 * c);
                    if (!PREFIX) {
                        // keys up to the row's position, and behind its window's lower end or among the first tokens
                        const int v = j * AT_TILE + col0 + 32 * c, a = it.lo - it.head + v;
                        const uint32_t in = p.window ? column_bits(t - p.window + 1 - a, 32) | column_bits(0, p.sinks - a) : 0xFFFFFFFFu;
                        uint32_t keys = in & column_bits(0, t + 1 - a);
                        if (v < it.head) keys = (keys & ~column_bits(0, it.head - v)) | column_bits(0, p.sinks - v);
                        bits &= real ? keys : 0u;
                    }
                    return bits;
                };
                bool formed = false;                      // the tile's weights
                uint32_t w[32];
                if (known && (width & 15) == 0) {
                    // every row has a reference
                    const bool full = j >= fa && j < fz;
                    const f32x2 r2 = pk(-m, -m);
                    f32x2 z = 0ull;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t r[32];
                        tc::tmem_ld32(s_t + col0 + 32 * c, r);
                        tc::tmem_ld_wait32(r);
                        if (!full) {
                            const uint32_t bits = seen(c);
                            if (__any_sync(0xffffffffu, bits != 0xFFFFFFFFu)) {
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (!(bits >> e & 1u)) r[e] = 0xFF800000u;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const f32x2 y = fma2(pk(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])), c2, r2);
                            float a, b2;
                            upk(y, a, b2);
                            a = ex2(a);
                            b2 = ex2(b2);
                            z = add2(z, pk(a, b2));
                            w[16 * c + e] = pack_bf16(a, b2);
                        }
                    }
                    // The weights may not add up to more than 2^32, and those of an item's first tile add up to something; a logit
                    // that is not a number sends the tile the other way, too, where it spreads.  (What lies behind a sequence's queries has
                    // no say in it: results do not depend on that.)
                    const float zs = sum2(z);
                    if (!any(late || (real && (!(zs <= AT_WEIGHT_MAX) || (!started && zs < AT_WEIGHT_MIN))))) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) tmem_st16(s_t + col0 + 16 * c, *reinterpret_cast<const uint32_t(*)[16]>(w + 16 * c));
                        l2 = add2(l2, z);
                        formed = true;
                    }
                }
                if (!formed) {
                    const int nch = min(2, max(0, width - col0 + 31) >> 5);
                    auto load = [&](uint32_t (&r)[32], int c) {
                        tc::tmem_ld32(s_t + col0 + 32 * c, r);
                        const uint32_t bits = seen(c);
                        tc::tmem_ld_wait32(r);
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!(bits >> e & 1u)) r[e] = 0xFF800000u;
                    };
                    if (!started) m = real ? -INFINITY : 0.f;            // (rows that are none have a reference)
                    float mx = -INFINITY;
#pragma unroll 1
                    for (int c = 0; c < nch; ++c) {
                        uint32_t r[32];
                        load(r, c);
#pragma unroll
                        for (int e = 0; e < 32; e += 2) mx = fmaxf(mx, fmaxf(__uint_as_float(r[e]), __uint_as_float(r[e + 1])));
                    }
                    sm_row[half][x][row] = mx;
                    if (any(late)) { dead = true; break; }
                    mx = __fmul_rn(fmaxf(mx, sm_row[half ^ 1][x][row]), p.c);
                    // (a maximum below the reference changes nothing)
                    if (!started) {
                        m = fmaxf(m, mx);
                    } else if (any(real && mx > m + AT_RAISE)) {
                        const float f = mx > m ? ex2(m - mx) : 1.f;
                        m = fmaxf(m, mx);
                        l2 = mul2(l2, pk(f, f));
#pragma unroll 1
                        for (int c = 0; c < D / 64; ++c) {
                            uint32_t o[32];
                            const uint32_t at = o_t + half * (D / 2) + 32 * c;
                            tc::tmem_ld32(at, o);
                            tc::tmem_ld_wait32(o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            tc::tmem_st32(at, o);
                        }
                    }
                    const float ref = m == -INFINITY ? 0.f : -m;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if (c >= nch) continue;
                        uint32_t r[32];
                        load(r, c);
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            // (scaled, rounded and then subtracted, as the maximum was: of logits beyond 2^24 a fused product's exact
                            // difference from a rounded reference may be anything.  Not mul2 and add2, which the assembler fuses.)
                            const float a = ex2(__fadd_rn(__fmul_rn(__uint_as_float(r[2 * e]), p.c), ref));
                            const float b2 = ex2(__fadd_rn(__fmul_rn(__uint_as_float(r[2 * e + 1]), p.c), ref));
                            l2 = add2(l2, pk(a, b2));
                            w[16 * c + e] = pack_bf16(a, b2);
                        }
                    }
                    const uint32_t nv = n + 2 * (j - jb) + 1, slot_v = nv % SLOTS;
                    const bool tail = width & 15, late_v = tail && !tc::mbar_wait(&bar_full[slot_v], (nv / SLOTS) & 1u, wc);
                    // (where every row has a reference from now on, the straight path takes over - but for references so large that its
                    // fused products would differ from this path's rounded ones by more than weights are rounded by)
                    known = !any((real && !(fabsf(m) <= AT_FUSED_MAX)) || late_v);
                    if (tail && any(late_v)) {
                        tc::tmem_st_wait();               // (O may be on its way back)
                        dead = true;
                        break;
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        if (c < nch) tmem_st16(s_t + col0 + 16 * c, *reinterpret_cast<const uint32_t(*)[16]>(w + 16 * c));
                    if (tail) {
                        // rows of V behind the last key, up to the next multiple of 16, may hold anything: cleared (by the warps of
                        // both query tiles, each before its own product)
                        uint8_t *v = ring + slot_v * SLOT_BYTES;
                        for (int e = (sw & 7) * 32 + lane; e < ((width + 15) / 16 * 16 - width) * 8 * NB; e += 256) {
                            const int vr = width + e / (8 * NB), vc = e % (8 * NB);
                            *reinterpret_cast<uint4 *>(v + (vc >> 3) * BLOCK + vr * 128 + (vc & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                        }
                        tc::fence_async_smem();
                    }
                }
                started = true;
                tc::tmem_st_wait();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&bar_p[x]);
            }
            if (dead) break;
            n += 2 * (je - jb);
            float l = sum2(l2);
            sm_row[half][x][row] = l;
            if (any(started && !tc::mbar_wait(&bar_o[x], no & 1u, wc))) break;
            l = half ? sm_row[0][x][row] + l : l + sm_row[1][x][row];
            no += started ? 1 : 0;
            const float inv = l == 0.f ? 0.f : 1.f / l, lse2 = l == 0.f ? -INFINITY : m + log2f(l);
            const int g = row_g, i = im.fi[x] + row_i, b = im.fb[x] + row_b;
            const long long R = (((long long)b * p.kv_heads + im.h) * p.n_q + i) * p.G + g;
            const bool last = p.slots == 1;
            const long long at = (long long)(PREFIX ? im.part : p.p_slots + im.part) * p.rows_total + R;
            // each of a row's threads stores half of its channels, 32 bytes at a time
            const long long to = (last ? b * p.os[0] + (long long)(im.h * p.G + g) * p.os[1] + (long long)i * p.os[2] : at * D) + half * (D / 2);
#pragma unroll 1
            for (int c = 0; c < D / 2; c += 16) {
                uint32_t o[16], u[8];
                tmem_ld16(o_t + half * (D / 2) + c, o);          // (whatever lies there, where there was nothing to add up)
                tmem_ld_wait16(o);
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = l == 0.f ? 0u : __float_as_uint(__uint_as_float(o[k]) * inv);
                if (real && last) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) u[k] = pack_bf16(__uint_as_float(o[2 * k]), __uint_as_float(o[2 * k + 1]));
                    store32(static_cast<__nv_bfloat16 *>(p.out) + to + c, u, wide);
                } else if (real && l != 0.f) {
#pragma unroll
                    for (int e = 0; e < 16; e += 8) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) u[k] = o[e + k];
                        store32(p.part_o + to + c + e, u, true);
                    }
                }
            }
            if (started) {
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&bar_o_read[x]);
            }
            if (real && half == 0) {
                if (!last) p.part_lse[at] = lse2;
                else if (p.lse_out) p.lse_out[((long long)b * p.kv_heads * p.G + im.h * p.G + g) * p.n_q + i] = natural_lse(lse2);
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bar_item_read[ni & 1u]);
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 0) tc::tmem_dealloc(tmem, 512);
    if (!first) pdl_wait();
}

}  // namespace obf
