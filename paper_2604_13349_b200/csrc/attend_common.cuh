// What the attention kernels over a relayed cache share: the call as they see it, which keys a run of query rows sees, where
// partial results go, and the kernel that joins them.
//
// A KV head's query rows are numbered r = i * G + g (query i, head g of the group), so that rows that see nearly the same keys
// are neighbours; over a shared prefix the rows of the whole batch are one run, r = (b * n_q + i) * G + g.  The keys that a run
// of rows sees are the first s and lo .. hi - 1; the kernels walk them as 0 .. s + hi - lo - 1 and cut that into `slots` equal
// parts when there are too few rows to fill the chip.  A part leaves out / lse of its keys alone, fp32, and the join weighs the
// parts by 2^(lse - common lse).
#pragma once

#include <climits>

#include "common.cuh"

namespace obf {

struct AttendDev {
    const void *q, *k, *v;
    void *out;
    long long qs[3], ks[3], vs[3], os[3];
    const void *pk, *pv;      // shared prefix, or null
    long long pks[2], pvs[2];
    const int32_t *lens, *q_lens;
    float *lse_out;
    const float *mass_in;
    float *mass_out;
    float decay;
    float c;                  // scale * log2 e: logits are kept in the log2 domain
    int32_t batch, kv_heads, G, n_q, capacity, window, sinks;
    int32_t prefix;           // rows of the shared prefix, 0 without one
    int32_t p_slots, slots;   // parts of the prefix and all parts of a row (own keys: slots - p_slots); 1: no join
    long long rows_total;     // batch * kv_heads * n_q * G
    // workspace
    uint32_t *status;
    float *part_o;            // [slots, rows_total, d]
    float *part_lse;          // [slots, rows_total], log2 domain, -inf: no keys (part_o is not written then)
    float *logits;            // [rows_total, capacity] when masses are asked for, visible keys only
    unsigned long long wait_limit_ns;
};

__device__ __forceinline__ int attend_len(const AttendDev &p, int b)
{
    const int n = p.lens ? p.lens[b] : p.capacity;
    return min(max(n, 0), p.capacity);
}

__device__ __forceinline__ int attend_q_len(const AttendDev &p, int b)
{
    const int n = p.q_lens ? p.q_lens[b] : p.n_q;
    return min(max(n, 0), p.n_q);
}

// The call's status word, by one block of its first kernel: whether a length had to be clamped.  Written, not ORed in, so that
// nothing of an earlier call is left in the workspace.
__device__ __forceinline__ void attend_status(const AttendDev &p)
{
    __shared__ uint32_t bad;
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
        const bool out = (p.lens && (p.lens[b] < 0 || p.lens[b] > p.capacity)) || (p.q_lens && (p.q_lens[b] < 0 || p.q_lens[b] > p.n_q));
        if (out) bad = OBF_DEV_INTERNAL;
    }
    __syncthreads();
    if (threadIdx.x == 0) *p.status = bad;
}

// Keys that queries at positions t0 .. t1 (t0 <= t1) of a sequence see between them: rows 0 .. s - 1 and lo .. hi - 1.
struct KeyRange {
    int s, lo, hi;
    __device__ __forceinline__ int count() const { return s + hi - lo; }
    __device__ __forceinline__ int key(int v) const { return v < s ? v : v - s + lo; }
};

__device__ __forceinline__ KeyRange attend_range(const AttendDev &p, int t0, int t1, int len)
{
    KeyRange r;
    r.hi = max(0, min(t1 + 1, len));
    r.lo = p.window ? min(max(0, t0 - p.window + 1), r.hi) : 0;
    r.s = p.window ? min(p.sinks, r.lo) : 0;
    return r;
}

__device__ __forceinline__ bool attend_sees(const AttendDev &p, int t, int j)
{
    return j <= t && (p.window == 0 || j > t - p.window || j < p.sinks);
}

// Final result of a row: out rounded to its type and lse in the natural log.
__device__ __forceinline__ float natural_lse(float lse2) { return lse2 * 0.6931471805599453f; }

// 2^x by the special-function unit (2 ulp; results below 2^-126 become zero).
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Four neighbouring channels of a row, rounded to its type.
template <typename T>
__device__ __forceinline__ void store4(T *dst, float4 v)
{
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(dst) = v;
    } else {
        __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
        uint2 w;
        w.x = *reinterpret_cast<uint32_t *>(&a);
        w.y = *reinterpret_cast<uint32_t *>(&b);
        *reinterpret_cast<uint2 *>(dst) = w;
    }
}

// ---- join -------------------------------------------------------------------------------------------------
// Blocks 0 .. rows_total - 1: a row each, its parts dealt out to four warps, a lane D / 32 channels.  The blocks behind them
// (only where masses are asked for) own AJ_KEYS keys of a (sequence, KV head) each: they need the lse of the head's at most 64
// rows, which they work out from the parts themselves, so that masses do not wait for the rows' blocks.
// Bound by latency: a few kilobytes per row.
constexpr int AJ_NT = 128;
constexpr int AJ_KEYS = 512;

__device__ __forceinline__ float join_lse(const AttendDev &p, long long R)
{
    float m = -INFINITY;
    for (int i = 0; i < p.slots; ++i) m = fmaxf(m, p.part_lse[(long long)i * p.rows_total + R]);
    if (!(m > -INFINITY)) return m;                       // no key (or only NaN: fmaxf drops it, the sum below keeps it)
    float z = 0.f;
    for (int i = 0; i < p.slots; ++i) z += exp2f(p.part_lse[(long long)i * p.rows_total + R] - m);
    return m + log2f(z);
}

template <typename TIN, int D>
__global__ void __launch_bounds__(AJ_NT) k_attend_join(const __grid_constant__ AttendDev p)
{
    pdl_wait();
    __shared__ float sh[4][D + 2];
    const int rows_bh = p.n_q * p.G;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((long long)blockIdx.x < p.rows_total) {
        constexpr int C = D / 32;
        const long long R = blockIdx.x;
        const int bh = (int)(R / rows_bh), r = (int)(R - (long long)bh * rows_bh);
        const int b = bh / p.kv_heads, h = bh - b * p.kv_heads, i = r / p.G, g = r - i * p.G;
        if (i >= attend_q_len(p, b)) return;
        float m = -INFINITY, z = 0.f, o[C];
#pragma unroll
        for (int e = 0; e < C; ++e) o[e] = 0.f;
        for (int sl = warp; sl < p.slots; sl += 4) {
            const float l = p.part_lse[(long long)sl * p.rows_total + R];
            if (l == -INFINITY) continue;
            const float mn = fmaxf(m, l), f = exp2f(m - mn), w = exp2f(l - mn);
            const float *src = p.part_o + ((long long)sl * p.rows_total + R) * D + lane * C;
            z = z * f + w;
#pragma unroll
            for (int e = 0; e < C; ++e) o[e] = o[e] * f + w * src[e];
            m = mn;
        }
#pragma unroll
        for (int e = 0; e < C; ++e) sh[warp][lane * C + e] = o[e];
        if (lane == 0) { sh[warp][D] = m; sh[warp][D + 1] = z; }
        __syncthreads();
        const float M = fmaxf(fmaxf(sh[0][D], sh[1][D]), fmaxf(sh[2][D], sh[3][D]));
        float Z = 0.f, f[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) { f[w] = sh[w][D + 1] == 0.f ? 0.f : exp2f(sh[w][D] - M); Z += f[w] * sh[w][D + 1]; }
        const float inv = Z == 0.f ? 0.f : 1.f / Z;
        for (int e = threadIdx.x; e < D / 4; e += AJ_NT) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                v.x += f[w] * sh[w][4 * e]; v.y += f[w] * sh[w][4 * e + 1]; v.z += f[w] * sh[w][4 * e + 2]; v.w += f[w] * sh[w][4 * e + 3];
            }
            v.x *= inv; v.y *= inv; v.z *= inv; v.w *= inv;
            store4(static_cast<TIN *>(p.out) + b * p.os[0] + (long long)(h * p.G + g) * p.os[1] + (long long)i * p.os[2] + 4 * e, v);
        }
        if (p.lse_out && threadIdx.x == 0)
            p.lse_out[((long long)b * p.kv_heads * p.G + h * p.G + g) * p.n_q + i] = Z == 0.f ? -INFINITY : natural_lse(M + log2f(Z));
        return;
    }
    // masses
    __shared__ float lse[64];
    const int per = (p.capacity + AJ_KEYS - 1) / AJ_KEYS;
    const long long blk = (long long)blockIdx.x - p.rows_total;
    const int bh = (int)(blk / per), j0 = (int)(blk - (long long)bh * per) * AJ_KEYS;
    const int b = bh / p.kv_heads;
    const int len = attend_len(p, b), ql = attend_q_len(p, b);
    if (j0 >= len) return;
    const int rows = ql * p.G;
    for (int r = threadIdx.x; r < rows; r += AJ_NT) lse[r] = join_lse(p, (long long)bh * rows_bh + r);
    __syncthreads();
    for (int j = j0 + threadIdx.x; j < min(j0 + AJ_KEYS, len); j += AJ_NT) {
        float sum = 0.f;
        for (int i = 0; i < ql; ++i) {
            if (!attend_sees(p, len - ql + i, j)) continue;
            for (int g = 0; g < p.G; ++g) {
                const int r = i * p.G + g;
                sum += exp2f(p.logits[((long long)bh * rows_bh + r) * p.capacity + j] - lse[r]);
            }
        }
        const long long at = (long long)bh * p.capacity + j;
        p.mass_out[at] = (p.mass_in ? p.decay * p.mass_in[at] : 0.f) + sum;
    }
}

}  // namespace obf
