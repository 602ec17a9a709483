// Attention of few query rows per KV head over a bf16 cache (decoding): bound by the reads of keys and values.
//
// A block of four warps owns a tile of 8 NT query rows and a part of the keys; each warp walks its own tiles of 16 keys through
// a private ring of stages in shared memory (16-byte asynchronous copies, rows past the end filled with zeros, 16-byte chunks
// swizzled by the row so that matrix loads meet every bank once), so warps never wait for one another before the end.  Keys lie
// on the M side of the 16 x 8 x 16 products: S^T = K Q^T and O^T += V^T P^T waste nothing for groups of up to eight rows, where
// queries on the M side would leave half of every product empty.  Two blocks share a multiprocessor: 128 KB
// and more of reads in flight; 4 sequences of up to 131072 keys 288 us (6.6 TB/s), 32 of up to 8192 with a window of 4096 75.1 us
// (6.0 TB/s).  Up to eight parts are a cluster, which joins them through shared memory and forms the masses of its own keys: one
// launch (one token over 1024 keys, window of 256: 5.4 us replayed from a graph).
//
// Softmax: a row's reference is its maximum at the time it was last raised; it is raised (and O and the sum rescaled) only when
// a logit exceeds it by more than 8 in the log2 domain, so weights stay below 2^8 and the common step has no shuffles.  Weights
// are rounded to bf16 for the second product, whose other operand is bf16 (off by at most 2^-8 of a weight; a bf16 output by 2.3e-3 of its
// norm where its own rounding alone makes 1.7e-3); the sum takes them in fp32.
#pragma once

#include "attend_common.cuh"

namespace obf {

constexpr int AF_WARPS = 4;
constexpr int AF_NT = 32 * AF_WARPS;
constexpr int AF_KEYS = 16;                               // keys of a stage
constexpr float AF_RAISE = 8.f;

template <int D>
constexpr int AF_STAGES = D == 128 ? 3 : 6;
template <int D>
constexpr int AF_STAGE_BYTES = 2 * AF_KEYS * D * 2;
template <int D>
__host__ __device__ constexpr size_t attend_few_smem() { return (size_t)AF_WARPS * AF_STAGES<D> * AF_STAGE_BYTES<D>; }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// ---- a cluster's blocks: meeting, and reading one another's shared memory ----
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_addr(const void *own, int rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(own)), "r"(rank));
    return r;
}
__device__ __forceinline__ float4 cluster_load4(uint32_t a)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float cluster_load(uint32_t a)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

// The end of a block with few rows: its warps' results, in shared memory, are weighed together and stored, or joined with those of
// the cluster's other blocks first.  osm: O as [warp][row][D + 4], ml: references and sums as [warp][row][2], room for one more
// result behind them.
template <int D, int ROWS>
__host__ __device__ constexpr size_t few_finish_smem() { return ((size_t)AF_WARPS * ROWS * (D + 4 + 2) + ROWS * (D + 4 + 1)) * 4; }

template <typename TIN, int D, int ROWS, bool PREFIX, bool CLUSTER>
__device__ __forceinline__ void few_finish(const AttendDev &p, const float *osm, float *ml, int tile, int part, int parts, int rows_run, int rows_seq, int h,
                                           int b_own, int len_own, int ql_own, const KeyRange &kr, int v0, int v1)
{
    auto locate_row = [&](int run, int &b, int &r) {
        b = PREFIX ? run / rows_seq : b_own;
        r = PREFIX ? run - b * rows_seq : run;
    };
    const bool last = p.slots == 1 && !p.mass_out;
    constexpr int TR = D / 4;                             // threads of a row, four channels each
    constexpr int LD = D + 4;
    float *cl = ml + AF_WARPS * ROWS * 2, *cl_lse = cl + ROWS * LD;       // what the cluster's other blocks read
    auto put = [&](int b, int h2, int i, int c, const float4 &a, float lse2) {
        store4(static_cast<TIN *>(p.out) + b * p.os[0] + (long long)h2 * p.os[1] + (long long)i * p.os[2] + c, a);
        if (p.lse_out && c == 0) p.lse_out[((long long)b * p.kv_heads * p.G + h2) * p.n_q + i] = natural_lse(lse2);
    };
    for (int row = threadIdx.x / TR; row < ROWS; row += AF_NT / TR) {
        const int run = tile * ROWS + row, c = threadIdx.x % TR * 4;
        int b, r;
        locate_row(run, b, r);
        const int i = r / p.G, g = r - i * p.G;
        if (run >= rows_run || i >= (PREFIX ? attend_q_len(p, b) : ql_own)) continue;
        float M = -INFINITY, Z = 0.f;
#pragma unroll
        for (int w = 0; w < AF_WARPS; ++w) M = fmaxf(M, ml[(w * ROWS + row) * 2]);
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < AF_WARPS; ++w) {
            const float z = ml[(w * ROWS + row) * 2 + 1], f = z == 0.f ? 0.f : exp2f(ml[(w * ROWS + row) * 2] - M);
            const float4 u = *reinterpret_cast<const float4 *>(&osm[(w * ROWS + row) * LD + c]);
            Z += f * z;
            a.x += f * u.x; a.y += f * u.y; a.z += f * u.z; a.w += f * u.w;
        }
        const float inv = Z == 0.f ? 0.f : 1.f / Z, lse2 = Z == 0.f ? -INFINITY : M + log2f(Z);
        a.x *= inv; a.y *= inv; a.z *= inv; a.w *= inv;
        if constexpr (CLUSTER) {
            *reinterpret_cast<float4 *>(&cl[row * LD + c]) = a;
            if (c == 0) cl_lse[row] = lse2;
        } else if (last) {
            put(b, h * p.G + g, i, c, a, lse2);
        } else {
            const long long at = (long long)(PREFIX ? part : p.p_slots + part) * p.rows_total + ((long long)b * p.kv_heads + h) * rows_seq + r;
            *reinterpret_cast<float4 *>(p.part_o + at * D + c) = a;
            if (c == 0) p.part_lse[at] = lse2;
        }
    }
    if constexpr (CLUSTER) {
        cluster_sync();
        for (int row = part + parts * (threadIdx.x / TR); row < ROWS; row += parts * (AF_NT / TR)) {
            const int r = tile * ROWS + row, c = threadIdx.x % TR * 4, i = r / p.G;
            if (r >= rows_run || i >= ql_own) continue;
            float l[8], M = -INFINITY, Z = 0.f;
            float4 u[8], a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < parts) {
                    l[k] = cluster_load(cluster_addr(cl_lse + row, k));
                    u[k] = cluster_load4(cluster_addr(cl + row * LD + c, k));
                    M = fmaxf(M, l[k]);
                }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < parts) {
                    const float f = l[k] == -INFINITY ? 0.f : exp2f(l[k] - M);
                    Z += f;
                    a.x += f * u[k].x; a.y += f * u[k].y; a.z += f * u[k].z; a.w += f * u[k].w;
                }
            const float inv = Z == 0.f ? 0.f : 1.f / Z;
            put(b_own, h * p.G + r - i * p.G, i, c, make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv), Z == 0.f ? -INFINITY : M + log2f(Z));
        }
        if (p.mass_out) {
            // Masses, in calls whose rows of a (sequence, KV head) are one tile: every block knows the lse of all rows now and adds up
            // the weights of its own keys, whose logits it has left in the workspace; of the keys that nobody sees it takes a share.
            __shared__ float lse[ROWS];
            const int rows = ql_own * p.G;
            if ((int)threadIdx.x < rows) {
                float l[8], M = -INFINITY, Z = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < parts) {
                        l[k] = cluster_load(cluster_addr(cl_lse + threadIdx.x, k));
                        M = fmaxf(M, l[k]);
                    }
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < parts) Z += l[k] == -INFINITY ? 0.f : exp2f(l[k] - M);
                lse[threadIdx.x] = M + log2f(Z);
            }
            __syncthreads();
            const long long bh = (long long)b_own * p.kv_heads + h;
            const float *x = p.logits + bh * rows_seq * p.capacity;
            const float *in = p.mass_in ? p.mass_in + bh * p.capacity : nullptr;
            float *out = p.mass_out + bh * p.capacity;
            for (int v = v0 + (int)threadIdx.x; v < v1; v += AF_NT) {
                const int j = kr.key(v);
                float sum = 0.f;
                for (int r = 0; r < rows; ++r)
                    if (attend_sees(p, len_own - ql_own + r / p.G, j)) sum += exp2f(x[(long long)r * p.capacity + j] - lse[r]);
                out[j] = (in ? p.decay * in[j] : 0.f) + sum;
            }
            const int e = (int)((long long)len_own * (part + 1) / parts);
            for (int j = (int)((long long)len_own * part / parts) + (int)threadIdx.x; j < e; j += AF_NT)
                if (!(j < kr.s || (j >= kr.lo && j < kr.hi))) out[j] = in ? p.decay * in[j] : 0.f;
        }
        cluster_sync();                                   // nobody leaves while its memory is read
    }
}

// CLUSTER: the parts of a tile, at most eight, are a cluster, which joins them through its shared memory; a shared prefix, in small
// calls, is walked as keys in front of each sequence's own.
template <int D, int NT, bool PREFIX, bool CLUSTER>
__global__ void __launch_bounds__(AF_NT) k_attend_few(const __grid_constant__ AttendDev p, const int first)
{
    static_assert(!(PREFIX && CLUSTER), "parts of a prefix are joined with those of the own keys");
    extern __shared__ __align__(128) unsigned char af_sm[];
    constexpr int KS = D / 16, CH = D / 8, ST = AF_STAGES<D>, ROWS = 8 * NT, LR = 32 / CH;
    // Behind the kernel of the shared prefix these blocks start as its make room: they read nothing of it, and what it waited for is
    // there.  Their own end waits for it, so that the join behind them sees both.
    if (first) pdl_wait();
    pdl_trigger();
    if (first && blockIdx.x == 0) attend_status(p);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rows_seq = p.n_q * p.G;
    const int rows_run = PREFIX ? p.batch * rows_seq : rows_seq, tiles = (rows_run + ROWS - 1) / ROWS;
    const int parts = PREFIX ? p.p_slots : p.slots - p.p_slots;
    unsigned x = blockIdx.x;
    const int part = x % parts;
    x /= parts;
    const int tile = x % tiles;
    x /= tiles;
    const int h = x % p.kv_heads, b_own = PREFIX ? 0 : x / p.kv_heads;
    const int len_own = PREFIX ? 0 : attend_len(p, b_own), ql_own = PREFIX ? 0 : attend_q_len(p, b_own);

    // keys that the tile's rows see
    KeyRange kr = {0, 0, 0};
    if (PREFIX) kr.hi = p.prefix;
    else {
        const int i0 = tile * ROWS / p.G, i1 = min((min((tile + 1) * ROWS, rows_seq) - 1) / p.G, ql_own - 1);
        if (i0 <= i1) kr = attend_range(p, len_own - ql_own + i0, len_own - ql_own + i1, len_own);
    }
    const int pre = CLUSTER ? p.with_prefix : 0;             // rows of the prefix walked before the own keys
    const int n = pre + kr.count(), per = ((n + 63) / 64 + parts - 1) / parts * 64;
    const int v0 = min((long long)part * per, (long long)n), v1 = min(v0 + per, n);

    const __nv_bfloat16 *kb = PREFIX ? static_cast<const __nv_bfloat16 *>(p.pk) + h * p.pks[0]
                                     : static_cast<const __nv_bfloat16 *>(p.k) + b_own * p.ks[0] + h * p.ks[1];
    const __nv_bfloat16 *vb = PREFIX ? static_cast<const __nv_bfloat16 *>(p.pv) + h * p.pvs[0]
                                     : static_cast<const __nv_bfloat16 *>(p.v) + b_own * p.vs[0] + h * p.vs[1];
    const long long kst = PREFIX ? p.pks[1] : p.ks[2], vst = PREFIX ? p.pvs[1] : p.vs[2];

    // this lane's share of a stage's copies: chunk lc of rows lr, lr + LR, ...
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(af_sm) + warp * ST * AF_STAGE_BYTES<D>;
    const int lc = lane % CH, lr = lane / CH;
    const int mine = (v1 - v0 + AF_KEYS - 1) / AF_KEYS;   // the part's stages, of which this warp does warp, warp + 4, ...
    auto fetch = [&](int st, int slot) {
        if (st < mine) {
            const uint32_t kd = ring + slot * AF_STAGE_BYTES<D>, vd = kd + AF_KEYS * D * 2;
            const int va = v0 + st * AF_KEYS;
#pragma unroll
            for (int i = 0; i < AF_KEYS / LR; ++i) {
                const int r = lr + i * LR, v = va + r;
                const bool real = v < v1;
                const int u = real ? v : v0;
                const uint32_t at = (uint32_t)(r * D * 2 + (lc ^ (r & 7)) * 16);
                if (CLUSTER && u < pre) {
                    cp_async16(kd + at, static_cast<const __nv_bfloat16 *>(p.pk) + h * p.pks[0] + u * p.pks[1] + lc * 8, real);
                    cp_async16(vd + at, static_cast<const __nv_bfloat16 *>(p.pv) + h * p.pvs[0] + u * p.pvs[1] + lc * 8, real);
                } else {
                    const long long j = kr.key(u - pre);
                    cp_async16(kd + at, kb + j * kst + lc * 8, real);
                    cp_async16(vd + at, vb + j * vst + lc * 8, real);
                }
            }
        }
        cp_commit();
    };
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) fetch(warp + s * AF_WARPS, s);

    // queries as B fragments, and the rows whose logits this lane holds: 8 nt + 2 (lane mod 4), + 1
    uint32_t qf[NT][KS][2];
    int row_t[NT][2];
    long long row_at[NT][2];
    auto locate_row = [&](int run, int &b, int &r) {
        b = PREFIX ? run / rows_seq : b_own;
        r = PREFIX ? run - b * rows_seq : run;
    };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int run = tile * ROWS + nt * 8 + lane / 4;
        int b, r;
        locate_row(run, b, r);
        const int i = r / p.G, g = r - i * p.G;
        const bool real = run < rows_run && i < (PREFIX ? attend_q_len(p, b) : ql_own);
        const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(p.q) + b * p.qs[0] + (long long)(h * p.G + g) * p.qs[1] + (long long)i * p.qs[2] + 2 * (lane & 3);
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e) qf[nt][k][e] = real ? *reinterpret_cast<const uint32_t *>(src + 16 * k + 8 * e) : 0u;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int run2 = tile * ROWS + nt * 8 + 2 * (lane & 3) + e;
            int b2, r2;
            locate_row(run2, b2, r2);
            const int i2 = r2 / p.G;
            row_t[nt][e] = INT_MIN;
            row_at[nt][e] = 0;
            if (run2 < rows_run && i2 < (PREFIX ? attend_q_len(p, b2) : ql_own)) {
                row_t[nt][e] = PREFIX ? INT_MAX : len_own - ql_own + i2;
                row_at[nt][e] = ((long long)b2 * p.kv_heads + h) * rows_seq + r2;
            }
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
    int slot = 0;
    for (int st = warp; st < mine; st += AF_WARPS) {
        cp_wait<ST - 2>();
        __syncwarp();
        // the slot that was read last is free again
        fetch(st + (ST - 1) * AF_WARPS, slot == 0 ? ST - 1 : slot - 1);
        const uint32_t kd = ring + slot * AF_STAGE_BYTES<D>, vd = kd + AF_KEYS * D * 2;
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
        {
            const int r = (lane & 7) + ((lane >> 3) & 1) * 8, c = lane >> 4;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint32_t a[4];
                ldsm4(a, kd + r * D * 2 + ((2 * k + c) ^ (r & 7)) * 16);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_bf16(s[nt], a, qf[nt][k][0], qf[nt][k][1]);
            }
        }
        // s[nt][2 u + e]: key 8 u + lane / 4 of the stage, row 8 nt + 2 (lane mod 4) + e
        const int va = v0 + st * AF_KEYS + lane / 4;
        bool raise = false;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int v = va + 8 * u, j = kr.key(v - pre);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const bool sees = v < v1 && (PREFIX || one_t || v < pre || attend_sees(p, row_t[nt][e], j));
                    float &y = s[nt][2 * u + e];
                    y = sees ? y * p.c : -INFINITY;
                    if (!PREFIX && p.mass_out && sees && row_t[nt][e] != INT_MIN) p.logits[row_at[nt][e] * p.capacity + j] = y;
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
        uint32_t pf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float r0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], r1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float w0 = ex2(s[nt][2 * u] - r0), w1 = ex2(s[nt][2 * u + 1] - r1);
                l[nt][0] += w0;
                l[nt][1] += w1;
                pf[nt][u] = transpose8x8(pack_bf16(w0, w1));
            }
        }
        {
            const int r = (lane & 7) + (lane >> 4) * 8, c = (lane >> 3) & 1;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint32_t a[4];
                ldsm4_t(a, vd + r * D * 2 + ((2 * k + c) ^ (r & 7)) * 16);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_bf16(o[nt][k], a, pf[nt][0], pf[nt][1]);
            }
        }
        slot = slot + 1 == ST ? 0 : slot + 1;
    }
    cp_wait<0>();
    __syncthreads();

    // the warps' results: O as [warp][row][D + 4], then references and sums
    constexpr int LD = D + 4;
    float *osm = reinterpret_cast<float *>(af_sm), *ml = osm + AF_WARPS * ROWS * LD;
    static_assert(few_finish_smem<D, ROWS>() <= attend_few_smem<D>(), "");
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float z = l[nt][e];
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) z += __shfl_xor_sync(0xffffffffu, z, w);
            const int row = 8 * nt + 2 * (lane & 3) + e;
            if (lane < 4) { ml[(warp * ROWS + row) * 2] = m[nt][e]; ml[(warp * ROWS + row) * 2 + 1] = z; }
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int u = 0; u < 2; ++u) osm[(warp * ROWS + row) * LD + 16 * k + 8 * u + lane / 4] = o[nt][k][2 * u + e];
        }
    __syncthreads();
    few_finish<__nv_bfloat16, D, ROWS, PREFIX, CLUSTER>(p, osm, ml, tile, part, parts, rows_run, rows_seq, h, b_own, len_own, ql_own, kr, v0, v1);
    if (!first) pdl_wait();
}

}  // namespace obf
