// Eviction by accumulated mass: selection and copy of the kept rows in one launch.
//
// A (sequence, KV head) is worked on by `parts` blocks.  Each finds the mass of the last row to keep by itself - a radix select
// over the order-preserving keys of the masses, 11 + 11 + 10 bits - walks the positions once, in order, to number the kept ones
// (slot = kept rows before it), and copies the rows of its own share of the slots.  Repeating the selection in every block
// costs reads of four bytes per position from the L2 cache and saves a launch and a trip through memory; sharing out slots, not
// positions, gives every block the same number of rows.  Bound by the copy: 2 rows read and written per kept position.
#pragma once

#include "attend_common.cuh"

namespace obf {

struct EvictDev {
    const void *k, *v;
    void *k_out, *v_out;
    long long ks[3], vs[3], kos[3], vos[3];      // bytes
    const float *mass;
    const int32_t *lens;
    int32_t *idx_out;
    float *mass_out;
    int32_t *lens_out;
    int32_t batch, kv_heads, capacity, keep, sinks, recent, mass_out_rows, parts;
};

constexpr int EM_NT = 512;
constexpr int EM_BINS = 2048;
constexpr int EM_LIST = 1024;                    // slots that a block numbers at a time
constexpr int EM_CACHE = 16384;                  // positions whose keys are kept in shared memory

constexpr size_t evict_smem(int capacity)
{
    return (size_t)(EM_BINS + EM_LIST + (capacity <= EM_CACHE ? (capacity + 3) / 4 * 4 : 0)) * 4;
}

// Larger mass, larger key; zeros of both signs are equal, NaN is below everything.
__device__ __forceinline__ uint32_t mass_key(float m) { return m == m ? score_key_bits(__float_as_uint(m + 0.f)) : 0u; }

template <int ROW_BYTES>
__global__ void __launch_bounds__(EM_NT) k_evict_mass(const __grid_constant__ EvictDev p)
{
    pdl_wait();
    extern __shared__ uint32_t em_sm[];
    uint32_t *hist = em_sm;
    int *list = reinterpret_cast<int *>(em_sm + EM_BINS);
    uint32_t *cache = em_sm + EM_BINS + EM_LIST;
    __shared__ uint32_t warp_tot[EM_NT / 32], found[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long bh = blockIdx.x / p.parts;
    const int part = (int)(blockIdx.x - bh * p.parts);
    const int b = (int)(bh / p.kv_heads), h = (int)(bh - (long long)b * p.kv_heads);
    const int len = p.lens ? min(max(p.lens[b], 0), p.capacity) : p.capacity;
    const int kept = min(p.keep, len);
    if (p.lens_out && part == 0 && h == 0 && tid == 0) p.lens_out[b] = kept;
    const int s0 = (int)((long long)kept * part / p.parts), s1 = (int)((long long)kept * (part + 1) / p.parts);
    if (s0 == s1) return;
    const float *mass = p.mass + bh * p.capacity;
    const bool cached = p.capacity <= EM_CACHE;
    const int c0 = p.sinks, c1 = len - p.recent;          // candidates, when not everything is kept
    uint32_t last = 0;                                    // key of the last candidate to keep
    int equal = 0;                                        // and how many of those with this key

    if (kept < len) {
        int want = kept - p.sinks - p.recent;
        if (want == 0) last = 0xFFFFFFFFu;
        if (cached)
            for (int j = c0 + tid; j < c1; j += EM_NT) cache[j] = mass_key(mass[j]);
        __syncthreads();
        uint32_t mask = 0;
        for (int pass = 0; pass < 3 && want > 0; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
            for (int i = tid; i < EM_BINS; i += EM_NT) hist[i] = 0;
            __syncthreads();
            for (int j = c0 + tid; j < c1; j += EM_NT) {
                const uint32_t k = cached ? cache[j] : mass_key(mass[j]);
                if ((k & mask) == last) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
            }
            __syncthreads();
            // how many lie in the bins above each: bins in falling order, four neighbours per thread
            uint32_t n[4], t = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) t += n[e] = hist[EM_BINS - 1 - (4 * tid + e)];
            uint32_t run = t;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += u;
            }
            if (lane == 31) warp_tot[warp] = run;
            __syncthreads();
            uint32_t above = run - t;
            for (int w = 0; w < warp; ++w) above += warp_tot[w];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (above < (uint32_t)want && above + n[e] >= (uint32_t)want) { found[0] = EM_BINS - 1 - (4 * tid + e); found[1] = above; }
                above += n[e];
            }
            __syncthreads();
            last |= found[0] << shift;
            mask |= (uint32_t)(bins - 1) << shift;
            want -= (int)found[1];
            __syncthreads();
        }
        equal = want;
    }

    const char *kb = static_cast<const char *>(p.k) + b * p.ks[0] + h * p.ks[1], *vb = static_cast<const char *>(p.v) + b * p.vs[0] + h * p.vs[1];
    char *ko = static_cast<char *>(p.k_out) + b * p.kos[0] + h * p.kos[1], *vo = static_cast<char *>(p.v_out) + b * p.vos[0] + h * p.vos[1];
    constexpr int CH = ROW_BYTES / 16;
    int at = 0, at_more = 0, at_same = 0;                 // where the sweep goes on: a position, and how many before it are kept for
                                                          // certain or have the last key
    for (int a = s0; a < s1; a += EM_LIST) {
        const int e1 = min(a + EM_LIST, s1);
        if (kept == len) {
            for (int i = a + tid; i < e1; i += EM_NT) list[i - a] = i;
        } else {
            int more = at_more, same = at_same;
            for (int j0 = at; j0 < len && more + min(same, equal) < e1; j0 += 4 * EM_NT) {
                at = j0;
                at_more = more;
                at_same = same;
                const int j = j0 + 4 * tid;
                uint32_t f[4], cnt = 0;                   // 1: kept for certain, 1 << 16: has the last key
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f[e] = 0;
                    if (j + e < len) {
                        if (j + e < c0 || j + e >= c1) f[e] = 1;
                        else {
                            const uint32_t k = cached ? cache[j + e] : mass_key(mass[j + e]);
                            f[e] = k > last ? 1u : k == last ? 1u << 16 : 0u;
                        }
                    }
                    cnt += f[e];
                }
                uint32_t run = cnt;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t u = __shfl_up_sync(0xffffffffu, run, o);
                    if (lane >= o) run += u;
                }
                __syncthreads();
                if (lane == 31) warp_tot[warp] = run;
                __syncthreads();
                uint32_t before = run - cnt, all = 0;
                for (int w = 0; w < EM_NT / 32; ++w) { if (w < warp) before += warp_tot[w]; all += warp_tot[w]; }
                int bm = more + (int)(before & 0xFFFFu), be = same + (int)(before >> 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int slot = bm + min(be, equal);
                    const bool take = f[e] == 1u || (f[e] != 0 && be < equal);
                    if (take && slot >= a && slot < e1) list[slot - a] = j + e;
                    bm += (int)(f[e] & 1u);
                    be += (int)(f[e] >> 16);
                }
                more += (int)(all & 0xFFFFu);
                same += (int)(all >> 16);
            }
        }
        __syncthreads();
        const int rows = e1 - a;
        for (int i = tid; i < rows; i += EM_NT) {
            const int j = list[i];
            if (p.idx_out) p.idx_out[bh * p.keep + a + i] = j;
            if (p.mass_out) p.mass_out[bh * p.mass_out_rows + a + i] = mass[j];
        }
        constexpr int U = 4, RS = EM_NT / CH;             // U rows of K and of V in flight per thread
        const int ch = (tid % CH) * 16;
        for (int i0 = tid / CH; i0 < rows; i0 += U * RS) {
            uint4 x[U], y[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * RS < rows) {
                    const long long j = list[i0 + u * RS];
                    x[u] = __ldcs(reinterpret_cast<const uint4 *>(kb + j * p.ks[2] + ch));
                    y[u] = __ldcs(reinterpret_cast<const uint4 *>(vb + j * p.vs[2] + ch));
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * RS < rows) {
                    const long long i = a + i0 + u * RS;
                    __stcs(reinterpret_cast<uint4 *>(ko + i * p.kos[2] + ch), x[u]);
                    __stcs(reinterpret_cast<uint4 *>(vo + i * p.vos[2] + ch), y[u]);
                }
        }
        __syncthreads();
    }
}

}  // namespace obf
