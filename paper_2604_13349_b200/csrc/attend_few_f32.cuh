// Attention of few query rows per KV head over an fp32 cache (decoding): bound by the reads of keys and values.
//
// As k_attend_few, on the CUDA cores: a block of four warps owns a tile of R = 4 or 8 query rows and a part of the keys.  D / 4 lanes
// share a key, four channels each, straight from global memory into registers, the next KEYS keys on their way while these are
// worked on.  A key's R products are summed over its lanes by trading halves - after log2 R steps every lane is left with the
// sum of one row - so R rows cost R - 1 + 5 - log2 R shuffles instead of 5 R; that lane forms the row's weight and the others
// fetch it for the second product.  References as in k_attend_few.  32 sequences of 8192 keys: 445 us (4.8 TB/s); with a window of
// 4096 over lengths of 1024 to 8192 238 us (3.7 TB/s).
#pragma once

#include "attend_few.cuh"

namespace obf {

template <int D, int R, bool PREFIX, bool CLUSTER>
__global__ void __launch_bounds__(AF_NT) k_attend_few_f32(const __grid_constant__ AttendDev p, const int first)
{
    constexpr int W = D / 4, GROUPS = 32 / W, KEYS = 4, STEP = GROUPS * KEYS;      // lanes of a key, keys side by side, keys of a lane, keys of a turn
    __shared__ __align__(16) float fin[few_finish_smem<D, R>() / 4];
    if (first) pdl_wait();                               // (else as in k_attend_few)
    pdl_trigger();
    if (first && blockIdx.x == 0) attend_status(p);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wl = lane % W, grp = lane / W;
    const int rows_seq = p.n_q * p.G;
    const int rows_run = PREFIX ? p.batch * rows_seq : rows_seq, tiles = (rows_run + R - 1) / R;
    const int parts = PREFIX ? p.p_slots : p.slots - p.p_slots;
    unsigned x = blockIdx.x;
    const int part = x % parts;
    x /= parts;
    const int tile = x % tiles;
    x /= tiles;
    const int h = x % p.kv_heads, b_own = PREFIX ? 0 : x / p.kv_heads;
    const int len_own = PREFIX ? 0 : attend_len(p, b_own), ql_own = PREFIX ? 0 : attend_q_len(p, b_own);
    KeyRange kr = {0, 0, 0};
    if (PREFIX) kr.hi = p.prefix;
    else {
        const int i0 = tile * R / p.G, i1 = min((min((tile + 1) * R, rows_seq) - 1) / p.G, ql_own - 1);
        if (i0 <= i1) kr = attend_range(p, len_own - ql_own + i0, len_own - ql_own + i1, len_own);
    }
    const int pre = CLUSTER ? p.with_prefix : 0;         // (as in k_attend_few)
    const int n = pre + kr.count(), per = ((n + 63) / 64 + parts - 1) / parts * 64;
    const int v0 = min((long long)part * per, (long long)n), v1 = min(v0 + per, n);
    const float *kb = (PREFIX ? static_cast<const float *>(p.pk) + h * p.pks[0] : static_cast<const float *>(p.k) + b_own * p.ks[0] + h * p.ks[1]) + 4 * wl;
    const float *vb = (PREFIX ? static_cast<const float *>(p.pv) + h * p.pvs[0] : static_cast<const float *>(p.v) + b_own * p.vs[0] + h * p.vs[1]) + 4 * wl;
    const long long kst = PREFIX ? p.pks[1] : p.ks[2], vst = PREFIX ? p.pvs[1] : p.vs[2];

    // keys va + grp + GROUPS e of a turn that begins at va
    ulonglong2 kn[KEYS], vn[KEYS];
    auto fetch = [&](int va) {
#pragma unroll
        for (int e = 0; e < KEYS; ++e) {
            const int v = va + grp + GROUPS * e;
            kn[e] = vn[e] = make_ulonglong2(0ull, 0ull);
            if (v < v1) {
                const long long j = kr.key(v - pre);
                const float *ka = kb + j * kst, *va2 = vb + j * vst;
                if (CLUSTER && v < pre) {
                    ka = static_cast<const float *>(p.pk) + h * p.pks[0] + v * p.pks[1] + 4 * wl;
                    va2 = static_cast<const float *>(p.pv) + h * p.pvs[0] + v * p.pvs[1] + 4 * wl;
                }
                kn[e] = __ldcs(reinterpret_cast<const ulonglong2 *>(ka));
                vn[e] = __ldcs(reinterpret_cast<const ulonglong2 *>(va2));
            }
        }
    };
    fetch(v0 + warp * STEP);

    // this lane's channels of the rows' queries, and the row whose weights it forms
    auto locate_row = [&](int run, int &b, int &r) {
        b = PREFIX ? run / rows_seq : b_own;
        r = PREFIX ? run - b * rows_seq : run;
    };
    ulonglong2 q[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int run = tile * R + k;
        int b, r;
        locate_row(run, b, r);
        const int i = r / p.G, g = r - i * p.G;
        q[k] = make_ulonglong2(0ull, 0ull);
        if (run < rows_run && i < (PREFIX ? attend_q_len(p, b) : ql_own))
            q[k] = *reinterpret_cast<const ulonglong2 *>(static_cast<const float *>(p.q) + b * p.qs[0] + (long long)(h * p.G + g) * p.qs[1] + (long long)i * p.qs[2] + 4 * wl);
    }
    constexpr int SHARE = W / R;                         // lanes left with the same row
    const int my = wl / SHARE;
    int t = INT_MIN;
    long long at = 0;
    {
        const int run = tile * R + my;
        int b, r;
        locate_row(run, b, r);
        const int i = r / p.G;
        if (run < rows_run && i < (PREFIX ? attend_q_len(p, b) : ql_own)) {
            t = PREFIX ? INT_MAX : len_own - ql_own + i;
            at = (((long long)b * p.kv_heads + h) * rows_seq + r) * p.capacity;
        }
    }
    const bool one_t = p.n_q == 1;
    float m = -INFINITY, l = 0.f;
    f32x2 o[R][2];
#pragma unroll
    for (int k = 0; k < R; ++k) o[k][0] = o[k][1] = 0ull;
    for (int va = v0 + warp * STEP; va < v1; va += AF_WARPS * STEP) {
        ulonglong2 kk[KEYS], vv[KEYS];
#pragma unroll
        for (int e = 0; e < KEYS; ++e) { kk[e] = kn[e]; vv[e] = vn[e]; }
        fetch(va + AF_WARPS * STEP);
        float s[KEYS];
        bool raise = false;
#pragma unroll
        for (int e = 0; e < KEYS; ++e) {
            float d[R];
#pragma unroll
            for (int k = 0; k < R; ++k) d[k] = sum2(fma2(q[k].y, kk[e].y, mul2(q[k].x, kk[e].x)));
            int off = W / 2;
#pragma unroll
            for (int c = R / 2; c >= 1; c /= 2, off /= 2) {
                const bool hi = wl & off;
#pragma unroll
                for (int k = 0; k < c; ++k) {
                    const float give = hi ? d[k] : d[k + c], keep = hi ? d[k + c] : d[k];
                    d[k] = keep + __shfl_xor_sync(0xffffffffu, give, off);
                }
            }
#pragma unroll
            for (; off >= 1; off /= 2) d[0] += __shfl_xor_sync(0xffffffffu, d[0], off);
            const int v = va + grp + GROUPS * e, j = kr.key(v - pre);
            const bool sees = v < v1 && (PREFIX || one_t || v < pre || attend_sees(p, t, j));
            s[e] = sees ? d[0] * p.c : -INFINITY;
            if (!PREFIX && p.mass_out && sees && t != INT_MIN && wl % SHARE == 0) p.logits[at + j] = s[e];
            raise = raise || s[e] > m + AF_RAISE;
        }
        if (__any_sync(0xffffffffu, raise)) {
            float mx = m;
#pragma unroll
            for (int e = 0; e < KEYS; ++e) mx = fmaxf(mx, s[e]);
            if (GROUPS == 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
            const float f = mx == -INFINITY ? 1.f : exp2f(m - mx);
            m = mx;
            l *= f;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float fk = __shfl_sync(0xffffffffu, f, k * SHARE, W);
                o[k][0] = mul2(o[k][0], pk(fk, fk));
                o[k][1] = mul2(o[k][1], pk(fk, fk));
            }
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int e = 0; e < KEYS; ++e) {
            const float w = exp2f(s[e] - ref);
            l += w;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float wk = __shfl_sync(0xffffffffu, w, k * SHARE, W);
                o[k][0] = fma2(pk(wk, wk), vv[e].x, o[k][0]);
                o[k][1] = fma2(pk(wk, wk), vv[e].y, o[k][1]);
            }
        }
    }
    // the two keys side by side are added up (they have the same references), then the warps' results go where few_finish looks
    constexpr int LD = D + 4;
    float *osm = fin, *ml = osm + AF_WARPS * R * LD;
    if (GROUPS == 2) l += __shfl_xor_sync(0xffffffffu, l, 16);
#pragma unroll
    for (int k = 0; k < R; ++k) {
        float4 a;
        upk(o[k][0], a.x, a.y);
        upk(o[k][1], a.z, a.w);
        if (GROUPS == 2) {
            a.x += __shfl_xor_sync(0xffffffffu, a.x, 16);
            a.y += __shfl_xor_sync(0xffffffffu, a.y, 16);
            a.z += __shfl_xor_sync(0xffffffffu, a.z, 16);
            a.w += __shfl_xor_sync(0xffffffffu, a.w, 16);
        }
        if (grp == 0) *reinterpret_cast<float4 *>(&osm[(warp * R + k) * LD + 4 * wl]) = a;
    }
    if (grp == 0 && wl % SHARE == 0) {
        ml[(warp * R + my) * 2] = m;
        ml[(warp * R + my) * 2 + 1] = l;
    }
    __syncthreads();
    few_finish<float, D, R, PREFIX, CLUSTER>(p, osm, ml, tile, part, parts, rows_run, rows_seq, h, b_own, len_own, ql_own, kr, v0, v1);
    if (!first) pdl_wait();
}

}  // namespace obf
