// Eviction by accumulated mass: selection and copy of the kept rows.
//
// Up to 16384 positions, one launch (k_evict_mass): a (sequence, KV head) is worked on by `parts` blocks.  Each finds the mass of
// the last row to keep by itself - its threads hold K neighbouring positions' keys in registers and count, bit by bit from the
// top, how many are at least the threshold tried; no histogram, whose few hot bins would serialise - numbers the kept positions
// by one scan (slot = kept rows before it) and copies the rows of its own share of the slots.  Repeating the selection in every
// block costs some microseconds of arithmetic and no traffic; sharing out slots, not positions, gives every block as many rows.
// Longer caches, two launches: a block per (sequence, head) selects by histograms of the keys, 11 + 11 + 10 bits, and writes the
// positions (k_evict_select); blocks over slots copy (k_evict_copy).
// Bound by the copy: 2 rows read and written per kept position.  32 x 8 caches of 3001 to 8192 rows to 2048: 112 us (4.9 TB/s), 12 of
// them the selection; 8 x 8 of 32768 to 16384 in two launches 220 us (5.0 TB/s).
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
constexpr int EM_CACHE = 32 * EM_NT;             // positions whose keys a block's registers hold
constexpr int ES_NT = 1024;
constexpr int ES_BINS = 2048;
constexpr int EC_ROWS = 256;                     // slots of a block of the copy

// Larger mass, larger key; zeros of both signs are equal, NaN is below everything.
__device__ __forceinline__ uint32_t mass_key(float m) { return m == m ? score_key_bits(__float_as_uint(m + 0.f)) : 0u; }

__device__ __forceinline__ int evict_len(const EvictDev &p, int b) { return p.lens ? min(max(p.lens[b], 0), p.capacity) : p.capacity; }

// Exclusive sums over a block's threads; `all`: the total.  `tot` holds a value per warp.
template <int NT>
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *tot, uint32_t &all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t run = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += u;
    }
    __syncthreads();
    if (lane == 31) tot[warp] = run;
    __syncthreads();
    const uint32_t w = lane < NT / 32 ? tot[lane] : 0u;
    all = __reduce_add_sync(0xffffffffu, w);
    return run - v + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0u);
}

// Copies rows list[0 .. rows) of a head to slots first .. of its outputs.
template <int ROW_BYTES, int NT>
__device__ __forceinline__ void evict_copy(const EvictDev &p, int b, int h, const int *list, int first, int rows)
{
    const char *kb = static_cast<const char *>(p.k) + b * p.ks[0] + h * p.ks[1], *vb = static_cast<const char *>(p.v) + b * p.vs[0] + h * p.vs[1];
    char *ko = static_cast<char *>(p.k_out) + b * p.kos[0] + h * p.kos[1], *vo = static_cast<char *>(p.v_out) + b * p.vos[0] + h * p.vos[1];
    constexpr int CH = ROW_BYTES / 16, U = 4, RS = NT / CH;   // U rows of K and of V in flight per thread
    const int ch = (threadIdx.x % CH) * 16;
    for (int i0 = threadIdx.x / CH; i0 < rows; i0 += U * RS) {
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
                const long long i = first + i0 + u * RS;
                __stcs(reinterpret_cast<uint4 *>(ko + i * p.kos[2] + ch), x[u]);
                __stcs(reinterpret_cast<uint4 *>(vo + i * p.vos[2] + ch), y[u]);
            }
    }
}

template <int ROW_BYTES, int K>
__global__ void __launch_bounds__(EM_NT, 2) k_evict_mass(const __grid_constant__ EvictDev p)
{
    pdl_wait();
    pdl_trigger();
    __shared__ uint32_t tot[2][EM_NT / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long bh = blockIdx.x / p.parts;
    const int part = (int)(blockIdx.x - bh * p.parts);
    const int b = (int)(bh / p.kv_heads), h = (int)(bh - (long long)b * p.kv_heads);
    const int len = evict_len(p, b), kept = min(p.keep, len);
    if (p.lens_out && part == 0 && h == 0 && tid == 0) p.lens_out[b] = kept;
    const int s0 = (int)((long long)kept * part / p.parts), s1 = (int)((long long)kept * (part + 1) / p.parts);
    if (s0 == s1) return;
    const float *mass = p.mass + bh * p.capacity;
    int *idx = p.idx_out + bh * p.keep;

    const int c0 = p.sinks, c1 = len - p.recent, j0 = tid * K;     // candidates, when not everything is kept
    uint32_t key[K];
    uint32_t last = 0;                                             // key of the last candidate to keep
    int equal = 0;                                                 // and how many of those with this key
    if (kept < len) {
#pragma unroll
        for (int e = 0; e < K; ++e) {
            const int j = j0 + e;
            key[e] = j >= c0 && j < c1 ? mass_key(mass[j]) : 0u;
        }
        const int want = kept - p.sinks - p.recent;
        if (want == 0) last = 0xFFFFFFFFu;
        bool exact = want == 0;
        for (int bit = 31, turn = 0; bit >= 0 && !exact; --bit, turn ^= 1) {
            const uint32_t tried = last | 1u << bit;
            uint32_t n = 0;
#pragma unroll
            for (int e = 0; e < K; ++e) n += key[e] >= tried ? 1u : 0u;
            n = __reduce_add_sync(0xffffffffu, n);
            if (lane == 0) tot[turn][warp] = n;
            __syncthreads();
            n = __reduce_add_sync(0xffffffffu, lane < EM_NT / 32 ? tot[turn][lane] : 0u);
            if ((int)n >= want) last = tried;
            exact = (int)n == want;                                // exactly these: all with at least this key
        }
        if (exact && want > 0) --last;                             // (tried >= 1)
        auto flag = [&](int e) {                                       // 1: kept for certain, 1 << 16: has the last key
            const int j = j0 + e;
            if (j >= len) return 0u;
            if (j < c0 || j >= c1) return 1u;
            return key[e] > last ? 1u : key[e] == last ? 1u << 16 : 0u;
        };
        uint32_t cnt = 0;
#pragma unroll
        for (int e = 0; e < K; ++e) cnt += flag(e);
        uint32_t all;
        const uint32_t before = block_scan<EM_NT>(cnt, tot[0], all);
        equal = exact ? 0 : kept - (int)(all & 0xFFFFu);
        int bm = (int)(before & 0xFFFFu), be = (int)(before >> 16);
#pragma unroll
        for (int e = 0; e < K; ++e) {
            const uint32_t f = flag(e);
            const int slot = bm + min(be, equal);
            const bool take = f == 1u || (f != 0u && be < equal);
            if (take && slot >= s0 && slot < s1) idx[slot] = j0 + e;
            bm += (int)(f & 1u);
            be += (int)(f >> 16);
        }
    } else {
        for (int i = s0 + tid; i < s1; i += EM_NT) idx[i] = i;
    }
    __syncthreads();                                               // the block reads back what it wrote
    if (p.mass_out)
        for (int i = s0 + tid; i < s1; i += EM_NT) p.mass_out[bh * p.mass_out_rows + i] = mass[idx[i]];
    evict_copy<ROW_BYTES, EM_NT>(p, b, h, idx + s0, s0, s1 - s0);
}

// Selection over a cache of any length, a block per (sequence, head): positions and masses of the kept rows.
__global__ void __launch_bounds__(ES_NT) k_evict_select(const __grid_constant__ EvictDev p)
{
    pdl_wait();
    pdl_trigger();
    __shared__ uint32_t hist[ES_BINS], tot[ES_NT / 32], found[2];
    const int tid = threadIdx.x;
    const long long bh = blockIdx.x;
    const int b = (int)(bh / p.kv_heads), h = (int)(bh - (long long)b * p.kv_heads);
    const int len = evict_len(p, b), kept = min(p.keep, len);
    if (p.lens_out && h == 0 && tid == 0) p.lens_out[b] = kept;
    const float *mass = p.mass + bh * p.capacity;
    const int c0 = p.sinks, c1 = len - p.recent;
    uint32_t last = 0;
    int equal = 0;
    auto keep_row = [&](int slot, int j) {
        p.idx_out[bh * p.keep + slot] = j;
        if (p.mass_out) p.mass_out[bh * p.mass_out_rows + slot] = mass[j];
    };
    if (kept == len) {
        for (int j = tid; j < len; j += ES_NT) keep_row(j, j);
        return;
    }
    int want = kept - p.sinks - p.recent;
    if (want == 0) last = 0xFFFFFFFFu;
    uint32_t mask = 0;
    for (int pass = 0; pass < 3 && want > 0; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
        for (int i = tid; i < ES_BINS; i += ES_NT) hist[i] = 0;
        __syncthreads();
#pragma unroll 4
        for (int j = c0 + tid; j < c1; j += ES_NT) {
            const uint32_t k = mass_key(mass[j]);
            if ((k & mask) == last) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
        }
        __syncthreads();
        // how many lie in the bins above each: bins in falling order, two neighbours per thread
        uint32_t n[2], all;
#pragma unroll
        for (int e = 0; e < 2; ++e) n[e] = hist[ES_BINS - 1 - (2 * tid + e)];
        uint32_t above = block_scan<ES_NT>(n[0] + n[1], tot, all);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (above < (uint32_t)want && above + n[e] >= (uint32_t)want) { found[0] = ES_BINS - 1 - (2 * tid + e); found[1] = above; }
            above += n[e];
        }
        __syncthreads();
        last |= found[0] << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        want -= (int)found[1];
        __syncthreads();
    }
    equal = want;
    int more = 0, same = 0;                                        // kept for certain, and with the last key, before the sweep's positions
    for (int j0 = 0; j0 < len && more + min(same, equal) < kept; j0 += 4 * ES_NT) {
        const int j = j0 + 4 * tid;
        uint32_t f[4], cnt = 0, all;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = 0;
            if (j + e < len) {
                if (j + e < c0 || j + e >= c1) f[e] = 1;
                else {
                    const uint32_t k = mass_key(mass[j + e]);
                    f[e] = k > last ? 1u : k == last ? 1u << 16 : 0u;
                }
            }
            cnt += f[e];
        }
        const uint32_t before = block_scan<ES_NT>(cnt, tot, all);
        int bm = more + (int)(before & 0xFFFFu), be = same + (int)(before >> 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (f[e] == 1u || (f[e] != 0u && be < equal)) keep_row(bm + min(be, equal), j + e);
            bm += (int)(f[e] & 1u);
            be += (int)(f[e] >> 16);
        }
        more += (int)(all & 0xFFFFu);
        same += (int)(all >> 16);
    }
}

template <int ROW_BYTES>
__global__ void __launch_bounds__(EM_NT) k_evict_copy(const __grid_constant__ EvictDev p)
{
    pdl_wait();
    pdl_trigger();
    __shared__ int list[EC_ROWS];
    const int per = (p.keep + EC_ROWS - 1) / EC_ROWS;
    const long long bh = blockIdx.x / per;
    const int a = (int)(blockIdx.x - bh * per) * EC_ROWS;
    const int b = (int)(bh / p.kv_heads), h = (int)(bh - (long long)b * p.kv_heads);
    const int rows = min(min(p.keep, evict_len(p, b)) - a, EC_ROWS);
    if (rows <= 0) return;
    for (int i = threadIdx.x; i < rows; i += EM_NT) list[i] = p.idx_out[bh * p.keep + a + i];
    __syncthreads();
    evict_copy<ROW_BYTES, EM_NT>(p, b, h, list, a, rows);
}

}  // namespace obf
