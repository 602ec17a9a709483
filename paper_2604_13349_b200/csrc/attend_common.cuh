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
#include <type_traits>

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
    int32_t cluster;          // the parts of a row are a cluster of blocks, which joins them
    int32_t with_prefix;      // rows of a prefix that each sequence's blocks read by themselves (small calls; `prefix` is 0 then)
    long long rows_total;     // batch * kv_heads * n_q * G
    // workspace
    uint32_t *status;
    float *part_o;            // [slots, rows_total, d]
    float *part_lse;          // [slots, rows_total], log2 domain, -inf: no keys (part_o is not written then)
    float *logits;            // [rows_total, capacity] when masses are asked for, visible keys only
    unsigned long long wait_limit_ns;
    int32_t debug_drop_load;  // OBF_FLAG_TEST_WAIT_EXPIRES
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

// Lets the stream's next kernel be set up while this one runs (it waits by itself for what it reads).  Behind pdl_wait(): what
// that kernel reads and this one does not write is there by then.
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- join -------------------------------------------------------------------------------------------------
// A row is joined by one warp where there are many rows, by the four warps of a block where there are few: a lane holds D / 32
// channels, its loads of the parts are independent of one another.  The blocks behind the rows' (only where masses are asked
// for) own AJ_KEYS keys of a (sequence, KV head) each; they work out the lse of the head's at most 64 rows from the parts
// themselves, so that masses do not wait for the rows' blocks.
// Bound by latency where the parts are few, else by reading them from the L2 cache.
constexpr int AJ_NT = 128;
constexpr int AJ_KEYS = 512;
constexpr int AJ_MAX_SLOTS = 256;

// Weights of a row's parts, the lanes of a warp working together: w[slot] = 2^(lse - common lse), and the common lse (log2).
// The weights add up to one; a row without keys gets zeros and -inf.
__device__ __forceinline__ float join_weights(const AttendDev &p, long long R, int lane, float *w)
{
    float m = -INFINITY, l[AJ_MAX_SLOTS / 32];
#pragma unroll
    for (int k = 0; k < AJ_MAX_SLOTS / 32; ++k) {
        const int sl = 32 * k + lane;
        l[k] = -INFINITY;
        if (32 * k >= p.slots) continue;
        if (sl < p.slots) l[k] = p.part_lse[(long long)sl * p.rows_total + R];
        m = fmaxf(m, l[k]);
    }
    m = warp_max(m);
    float z = 0.f;
#pragma unroll
    for (int k = 0; k < AJ_MAX_SLOTS / 32; ++k) {
        if (32 * k >= p.slots) continue;
        l[k] = l[k] == -INFINITY ? 0.f : exp2f(l[k] - m);          // (a lse that is not a number spreads, the maximum ignores it)
        z += l[k];
    }
    z = warp_sum(z);
    const float inv = z == 0.f ? 0.f : 1.f / z;
#pragma unroll
    for (int k = 0; k < AJ_MAX_SLOTS / 32; ++k)
        if (32 * k + lane < p.slots) w[32 * k + lane] = l[k] * inv;
    __syncwarp();
    return z == 0.f ? -INFINITY : m + log2f(z);
}

template <typename TIN, int D, int WARPS>
__global__ void __launch_bounds__(AJ_NT) k_attend_join(const __grid_constant__ AttendDev p, const int row_blocks)
{
    pdl_wait();
    pdl_trigger();
    constexpr int C = D / 32, ROWS = AJ_NT / 32 / WARPS;            // rows of a block
    typedef typename std::conditional<C == 4, float4, float2>::type vec;
    __shared__ float wt[4][AJ_MAX_SLOTS];
    __shared__ vec sh[4][32];
    const int rows_bh = p.n_q * p.G;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((int)blockIdx.x < row_blocks) {
        const long long R = (long long)blockIdx.x * ROWS + warp / WARPS;
        const bool there = R < p.rows_total;
        const int bh = there ? (int)(R / rows_bh) : 0, r = there ? (int)(R - (long long)bh * rows_bh) : 0;
        const int b = bh / p.kv_heads, h = bh - b * p.kv_heads, i = r / p.G, g = r - i * p.G;
        if (!there || i >= attend_q_len(p, b)) return;              // (the same in every warp of a row)
        const float lse2 = join_weights(p, R, lane, wt[warp]);
        float o[C];
#pragma unroll
        for (int e = 0; e < C; ++e) o[e] = 0.f;
        const float *src = p.part_o + R * D + lane * C;
#pragma unroll 8
        for (int sl = warp % WARPS; sl < p.slots; sl += WARPS) {
            const float w = wt[warp][sl];
            if (w == 0.f) continue;                                  // nothing was written there
            const vec v = *reinterpret_cast<const vec *>(src + (long long)sl * p.rows_total * D);
            o[0] += w * v.x;
            o[1] += w * v.y;
            if constexpr (C == 4) { o[2] += w * v.z; o[3] += w * v.w; }
        }
        if constexpr (WARPS > 1) {
            vec v;
            v.x = o[0];
            v.y = o[1];
            if constexpr (C == 4) { v.z = o[2]; v.w = o[3]; }
            sh[warp][lane] = v;
            __syncthreads();
            if (warp != 0) return;
#pragma unroll
            for (int e = 0; e < C; ++e) o[e] = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const vec u = sh[k][lane];
                o[0] += u.x;
                o[1] += u.y;
                if constexpr (C == 4) { o[2] += u.z; o[3] += u.w; }
            }
        }
        TIN *dst = static_cast<TIN *>(p.out) + b * p.os[0] + (long long)(h * p.G + g) * p.os[1] + (long long)i * p.os[2] + lane * C;
        if constexpr (C == 4) {
            store4(dst, make_float4(o[0], o[1], o[2], o[3]));
        } else if constexpr (sizeof(TIN) == 4) {
            *reinterpret_cast<float2 *>(dst) = make_float2(o[0], o[1]);
        } else {
            *reinterpret_cast<uint32_t *>(dst) = pack_bf16(o[0], o[1]);
        }
        if (p.lse_out && lane == 0) p.lse_out[((long long)b * p.kv_heads * p.G + h * p.G + g) * p.n_q + i] = natural_lse(lse2);
        return;
    }
    // masses
    __shared__ float lse[64];
    const int per = (p.capacity + AJ_KEYS - 1) / AJ_KEYS;
    const int blk = (int)blockIdx.x - row_blocks;
    const int bh = blk / per, j0 = (blk - bh * per) * AJ_KEYS;
    const int b = bh / p.kv_heads;
    const int len = attend_len(p, b), ql = attend_q_len(p, b);
    if (j0 >= len) return;
    const int rows = ql * p.G;
    constexpr int K = AJ_KEYS / AJ_NT;
    const long long at = (long long)bh * p.capacity + j0 + threadIdx.x;
    float in[K], sum[K];
#pragma unroll
    for (int e = 0; e < K; ++e) {
        sum[e] = 0.f;
        in[e] = p.mass_in && j0 + (int)threadIdx.x + e * AJ_NT < len ? p.mass_in[at + e * AJ_NT] : 0.f;
    }
    for (int r = warp; r < rows; r += AJ_NT / 32) {
        const float l = join_weights(p, (long long)bh * rows_bh + r, lane, wt[warp]);
        if (lane == 0) lse[r] = l;
    }
    __syncthreads();
    for (int i = 0; i < ql; ++i) {
        const int t = len - ql + i;
        bool sees[K];
#pragma unroll
        for (int e = 0; e < K; ++e) {
            const int j = j0 + (int)threadIdx.x + e * AJ_NT;
            sees[e] = j < len && attend_sees(p, t, j);
        }
        const float *x = p.logits + ((long long)bh * rows_bh + i * p.G) * p.capacity + j0 + threadIdx.x;
#pragma unroll 4
        for (int g = 0; g < p.G; ++g) {
#pragma unroll
            for (int e = 0; e < K; ++e)
                if (sees[e]) sum[e] += exp2f(x[(long long)g * p.capacity + e * AJ_NT] - lse[i * p.G + g]);
        }
    }
#pragma unroll
    for (int e = 0; e < K; ++e)
        if (j0 + (int)threadIdx.x + e * AJ_NT < len) p.mass_out[at + e * AJ_NT] = p.decay * in[e] + sum[e];
}

}  // namespace obf
