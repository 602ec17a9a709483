// Attention over a relayed cache on the CUDA cores: fp32 caches with more than 16 query rows per KV head, and bf16 where the
// tensor-core kernels do not apply or the caller asks for these.
//
// A block owns 64 query rows of a KV head and a part of their keys, in tiles of 64: logits as 4 x 4 register tiles of dot
// products (tile_dots), a running maximum and sum per row, the weights over the tile of keys in shared memory, and 4 rows x D / 16
// channels of the output per thread, two channels per multiply-add.  All in fp32.  Bound by the multiply-adds and the shared-memory
// reads that feed them (a 16-byte read costs four cycles of the shared-memory path also where the lanes read the same): 32 TFLOP/s on
// a causal fp32 prompt of 4096 with heads of 64 channels (28 before the next tile was copied ahead), 21 with a window of 300, where 512
// blocks of five tiles each make two rounds of 296.  8 x 2 and 8 x 4 logits per thread measured 30 and 29: the one reads as much per
// multiply-add, the other leaves half the warps to cover the latencies.
#pragma once

#include "attend_few.cuh"

namespace obf {

constexpr int AG_NT = 256;
constexpr int AG_TILE = 64;

// fp32 heads of 64 channels: the next tile of keys and values is copied while this one is worked on.
template <typename TIN, int D>
constexpr bool AG_ASYNC = sizeof(TIN) == 4 && D == 64;
template <typename TIN, int D>
constexpr size_t attend_generic_smem() { return (size_t)((AG_ASYNC<TIN, D> ? 5 : 3) * AG_TILE * TD_LD<D>) * sizeof(float); }
static_assert(TD_LD<64> >= AG_TILE + 4, "the weights lie over the keys");

__device__ __forceinline__ float4 scaled(f32x2 a, f32x2 b, float f)
{
    float4 v;
    upk(a, v.x, v.y);
    upk(b, v.z, v.w);
    return make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
}

// One of the call's two sets of keys: the sequences' own ones (PREFIX false) or the shared prefix.
template <typename TIN, int D, bool PREFIX>
__global__ void __launch_bounds__(AG_NT, 2) k_attend_generic(const __grid_constant__ AttendDev p, const int first)
{
    if (first) pdl_wait();                               // (else as in k_attend_few)
    pdl_trigger();
    extern __shared__ float sm[];
    constexpr int TILE = AG_TILE * TD_LD<D>;
    constexpr bool ASYNC = AG_ASYNC<TIN, D>;
    float *Qs = sm, *Ks = Qs + TILE, *Vs = Ks + TILE;
    constexpr int P_LD = AG_TILE + 4, VEC = 16 / sizeof(TIN), CH = D / VEC, CT = D / 16;
    __shared__ int row_t[AG_TILE];                       // position of a row's query, INT_MIN: not a query of the call
    __shared__ long long row_at[AG_TILE];                // its number among the call's rows
    if (first && blockIdx.x == 0) attend_status(p);

    const int parts = PREFIX ? p.p_slots : p.slots - p.p_slots;
    const int rows_seq = p.n_q * p.G;                    // rows of a (sequence, KV head)
    const long long rows_run = PREFIX ? (long long)p.batch * rows_seq : rows_seq;
    const int tiles = (int)((rows_run + AG_TILE - 1) / AG_TILE);
    long long x = blockIdx.x;
    const int part = (int)(x % parts);
    x /= parts;
    const int tile = tiles - 1 - (int)(x % tiles);       // the longest key ranges first
    x /= tiles;
    const int h = (int)(x % p.kv_heads), b_own = PREFIX ? 0 : (int)(x / p.kv_heads);

    // the rows
    for (int i = threadIdx.x; i < AG_TILE * CH; i += AG_NT) {
        const int rr = i / CH, ch = i - rr * CH;
        const long long run = (long long)tile * AG_TILE + rr;
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = 0.f;
        int t = INT_MIN;
        long long at = 0;
        if (run < rows_run) {
            const int b = PREFIX ? (int)(run / rows_seq) : b_own, r = (int)(run - (long long)(PREFIX ? b * (long long)rows_seq : 0));
            const int qi = r / p.G, g = r - qi * p.G, ql = attend_q_len(p, b);
            if (qi < ql) {
                t = attend_len(p, b) - ql + qi;
                at = ((long long)b * p.kv_heads + h) * rows_seq + r;
                const TIN *src = static_cast<const TIN *>(p.q) + b * p.qs[0] + (long long)(h * p.G + g) * p.qs[1] + (long long)qi * p.qs[2] + ch * VEC;
                unpack16<TIN>(*reinterpret_cast<const uint4 *>(src), f);
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) Qs[rr * TD_LD<D> + ch * VEC + e] = f[e];
        if (ch == 0) { row_t[rr] = t; row_at[rr] = at; }
    }
    __syncthreads();

    int t0 = INT_MAX, t1 = INT_MIN;                      // positions of the tile's first and last query
    bool whole = true;                                   // all its rows are queries
    for (int rr = 0; rr < AG_TILE; ++rr) {
        if (row_t[rr] == INT_MIN) { whole = false; continue; }
        t0 = min(t0, row_t[rr]);
        t1 = max(t1, row_t[rr]);
    }
    // the keys
    KeyRange kr;
    if (PREFIX) {
        kr.s = kr.lo = 0;
        kr.hi = p.prefix;
    } else {
        kr.s = kr.lo = kr.hi = 0;
        if (t1 != INT_MIN) kr = attend_range(p, t0, t1, attend_len(p, b_own));
    }
    const int n = kr.count();
    const int per = (int)(((long long)(n + AG_TILE - 1) / AG_TILE + parts - 1) / parts) * AG_TILE;
    const int v0 = min((long long)part * per, (long long)n), v1 = min((long long)v0 + per, (long long)n);
    const TIN *kb = PREFIX ? static_cast<const TIN *>(p.pk) + h * p.pks[0] : static_cast<const TIN *>(p.k) + b_own * p.ks[0] + h * p.ks[1];
    const TIN *vb = PREFIX ? static_cast<const TIN *>(p.pv) + h * p.pvs[0] : static_cast<const TIN *>(p.v) + b_own * p.vs[0] + h * p.vs[1];
    const long long kst = PREFIX ? p.pks[1] : p.ks[2], vst = PREFIX ? p.pvs[1] : p.vs[2];

    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    float m[4], l[4];
    f32x2 o[4][CT / 2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int e = 0; e < CT / 2; ++e) o[i][e] = 0ull;
    }
    auto fetch = [&](int v, float *kd, float *vd) {
        for (int i = threadIdx.x; i < AG_TILE * CH; i += AG_NT) {
            const int rr = i / CH, ch = i - rr * CH;
            const bool there = v + rr < v1;
            const long long j = kr.key(there ? v + rr : v0);
            const uint32_t at = (uint32_t)(rr * TD_LD<D> + ch * VEC) * 4;
            cp_async16((uint32_t)__cvta_generic_to_shared(kd) + at, kb + j * kst + ch * VEC, there);
            cp_async16((uint32_t)__cvta_generic_to_shared(vd) + at, vb + j * vst + ch * VEC, there);
        }
        cp_commit();
    };
    if (ASYNC && v0 < v1) fetch(v0, Ks, Vs);
    for (int v = v0, turn = 0; v < v1; v += AG_TILE, turn ^= 1) {
        __syncthreads();
        if constexpr (ASYNC) {
            // (the other buffers' last readers are through)
            Ks = Qs + TILE + 2 * turn * TILE;
            Vs = Ks + TILE;
            if (v + AG_TILE < v1) fetch(v + AG_TILE, Qs + TILE + 2 * (turn ^ 1) * TILE, Qs + 2 * TILE + 2 * (turn ^ 1) * TILE);
            else cp_commit();
            cp_wait<1>();
        } else
        for (int i = threadIdx.x; i < AG_TILE * CH; i += AG_NT) {
            const int rr = i / CH, ch = i - rr * CH;
            float f[VEC], w[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = w[e] = 0.f;
            if (v + rr < v1) {
                const int j = kr.key(v + rr);
                unpack16<TIN>(*reinterpret_cast<const uint4 *>(kb + j * kst + ch * VEC), f);
                unpack16<TIN>(*reinterpret_cast<const uint4 *>(vb + j * vst + ch * VEC), w);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) { Ks[rr * TD_LD<D> + ch * VEC + e] = f[e]; Vs[rr * TD_LD<D> + ch * VEC + e] = w[e]; }
        }
        __syncthreads();
        float s[4][4];
        tile_dots<D>(Qs, Ks, ty, tx, s);
        __syncthreads();                                 // the weights go where the keys were
        float *Ps = Ks;
        // whether every row sees every key of the tile (not asked for heads of 128 channels, whose registers are full)
        const int ja = kr.key(v), jb = kr.key(v + AG_TILE - 1);
        const bool full = D == 64 && whole && v + AG_TILE <= v1 && (PREFIX || ((v >= kr.s || v + AG_TILE <= kr.s) && jb <= t0 && (p.window == 0 || ja > t1 - p.window || jb < p.sinks)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = row_t[ty + 16 * i];
            float mx = m[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int vv = v + tx + 16 * e, j = vv < v1 ? kr.key(vv) : 0;
                const bool sees = full || (vv < v1 && t != INT_MIN && (PREFIX || attend_sees(p, t, j)));
                s[i][e] = sees ? s[i][e] * p.c : -INFINITY;
                if (!PREFIX && p.mass_out && sees) p.logits[row_at[ty + 16 * i] * p.capacity + j] = s[i][e];
                mx = fmaxf(mx, s[i][e]);
            }
#pragma unroll
            for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
            const float ref = mx == -INFINITY ? 0.f : mx, f = exp2f(m[i] - ref);
            float z = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float w = exp2f(s[i][e] - ref);
                Ps[(ty + 16 * i) * P_LD + tx + 16 * e] = w;
                z += w;
            }
            l[i] = l[i] * f + z;
            m[i] = mx;
#pragma unroll
            for (int e = 0; e < CT / 2; ++e) o[i][e] = mul2(o[i][e], pk(f, f));
        }
        __syncwarp();                                    // a row's weights are written and read by the same half warp
#pragma unroll 2
        for (int j = 0; j < AG_TILE; j += 2) {
            float pw[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 u = *reinterpret_cast<const float2 *>(&Ps[(ty + 16 * i) * P_LD + j]);
                pw[i][0] = u.x;
                pw[i][1] = u.y;
            }
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int e = 0; e < CT / 2; e += 2) {
                    const ulonglong2 w = *reinterpret_cast<const ulonglong2 *>(&Vs[(j + q) * TD_LD<D> + 4 * tx + 32 * e]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x2 pp = pk(pw[i][q], pw[i][q]);
                        o[i][e] = fma2(pp, w.x, o[i][e]);
                        o[i][e + 1] = fma2(pp, w.y, o[i][e + 1]);
                    }
                }
        }
        __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
        const int rr = ty + 16 * i;
        if (row_t[rr] == INT_MIN) continue;
        const long long R = row_at[rr];
        const float inv = l[i] == 0.f ? 0.f : 1.f / l[i], lse2 = l[i] == 0.f ? -INFINITY : m[i] + log2f(l[i]);
        if (p.slots == 1 && !p.mass_out) {
            const int bh = (int)(R / rows_seq), r = (int)(R - (long long)bh * rows_seq), b = bh / p.kv_heads, qi = r / p.G, hq = h * p.G + r - qi * p.G;
            TIN *dst = static_cast<TIN *>(p.out) + b * p.os[0] + (long long)hq * p.os[1] + (long long)qi * p.os[2];
#pragma unroll
            for (int e = 0; e < CT / 2; e += 2) store4(dst + 4 * tx + 32 * e, scaled(o[i][e], o[i][e + 1], inv));
            if (p.lse_out && tx == 0) p.lse_out[((long long)b * p.kv_heads * p.G + hq) * p.n_q + qi] = natural_lse(lse2);
        } else {
            const long long at = (long long)(PREFIX ? part : p.p_slots + part) * p.rows_total + R;
#pragma unroll
            for (int e = 0; e < CT / 2; e += 2) *reinterpret_cast<float4 *>(p.part_o + at * D + 4 * tx + 32 * e) = scaled(o[i][e], o[i][e + 1], inv);
            if (tx == 0) p.part_lse[at] = lse2;
        }
    }
    if (!first) pdl_wait();
}

}  // namespace obf
