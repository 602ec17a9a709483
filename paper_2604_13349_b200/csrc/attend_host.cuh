// Host-side helpers that the attention entry points share: checks of strides, the number of parts that keys are cut into, limits.
#pragma once

#include <climits>

#include "attend_common.cuh"
#include "host.cuh"

namespace obf {

// obf_attend for entry points of other files (obf_attend.cu): whether a call's queries are many enough for the tensor cores' tiles of 128 rows, its
// workspace, and the call itself, with a factor for each key's logits and weights where it goes to those tiles (AttendDev).
struct AttendFactors {
    const float4 *of;
    long long stride;
};
bool attends_in_tiles(const obf_attend_t *a);
size_t attend_rows_bytes(const obf_attend_t *a);
obf_status_t attend_rows(const obf_attend_t *a, const AttendFactors &factors, void *workspace, size_t bytes, void *stream);

inline obf_status_t check_stride(const int64_t *st, const int64_t *n, int dims, int head_dim, int esize)
{
    for (int i = 0; i < dims; ++i) {
        if (n[i] < 2) continue;                           // never stepped over
        if (st[i] < head_dim || st[i] >= ((int64_t)1 << 40) / esize || st[i] * esize % 16 != 0) return OBF_ERR_INVALID_ARG;
    }
    return OBF_OK;
}

// Parts of `keys` keys for `tiles` tiles of query rows: about `blocks` blocks in all, at least `least` keys each.
inline int parts_for(long long tiles, long long keys, long long blocks, int least)
{
    long long s = (blocks + tiles - 1) / tiles, most = (keys + least - 1) / least;
    if (s > most) s = most;
    if (s > 128) s = 128;
    return (int)(s < 1 ? 1 : s);
}

// Parts of the keys for k_attend_few: as many as make its rounds of resident blocks cheapest, a block costing its keys and, to
// begin and to end, as much as 120 more; at least 256 keys each.  (Measured beside one another: 16 sequences of 8192
// keys and their masses, 128 tiles: the rule's 9 parts 96 us, 18 parts 99, 28 parts 101; 32 of up to 8192 with a window of 4096: the rule's
// 1 part 74.6, 9 parts 80; 4 of 131072: the rule's 37 parts 283, 9 parts 286, 18 parts 281, 28 parts, whose last round is the emptiest, 292.)
inline int few_parts(long long tiles, long long keys, int resident)
{
    long long best = 1, cost = LLONG_MAX;
    for (long long s = 1; s <= 128 && (s == 1 || s * 256 <= keys); ++s) {
        const long long c = (tiles * s + resident - 1) / resident * ((keys + s - 1) / s + 120);
        if (c < cost) { cost = c; best = s; }
    }
    return (int)best;
}

// Keys that a query row can see at most.
inline long long most_keys(const obf_attend_t *a, int rows_of_queries)
{
    if (a->window == 0) return a->capacity;
    const long long n = (long long)a->window + rows_of_queries + a->sinks;
    return n < a->capacity ? n : a->capacity;
}

// Raises a kernel's shared-memory limit the first time it is used on a device.
template <typename K>
inline obf_status_t set_smem_once(K kernel, size_t bytes, bool (&done)[64])
{
    int dev = 0;
    OBF_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 0 && dev < 64 && done[dev]) return OBF_OK;
    OBF_TRY(set_smem(kernel, bytes));
    if (dev >= 0 && dev < 64) done[dev] = true;
    return OBF_OK;
}

template <typename TIN, int D>
inline obf_status_t launch_join(const AttendDev &p, cudaStream_t st)
{
    // a warp per row fills the chip from some thousand rows on; fewer are joined by four warps each
    const bool many = p.rows_total >= 4 * 148;
    const long long row_blocks = many ? (p.rows_total + 3) / 4 : p.rows_total;
    long long blocks = row_blocks;
    if (p.mass_out) blocks += (long long)p.batch * p.kv_heads * ((p.capacity + AJ_KEYS - 1) / AJ_KEYS);
    if (blocks > INT_MAX) return OBF_ERR_UNSUPPORTED;
    if (many) OBF_TRY(launch(k_attend_join<TIN, D, 1>, dim3((unsigned)blocks), AJ_NT, 0, st, p, (int)row_blocks));
    else OBF_TRY(launch(k_attend_join<TIN, D, 4>, dim3((unsigned)blocks), AJ_NT, 0, st, p, (int)row_blocks));
    ++g_last_launches;
    return OBF_OK;
}

}  // namespace obf
