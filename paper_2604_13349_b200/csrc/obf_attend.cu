// Host side of the operators on a relayed cache (include/obf.h): argument validation, workspace layout, kernel dispatch.
#include <cmath>

#include "attend_common.cuh"
#include "attend_few.cuh"
#include "attend_few_f32.cuh"
#include "attend_generic.cuh"
#include "attend_tc.cuh"
#include "evict_mass.cuh"
#include "host.cuh"

namespace obf {

static obf_status_t check_stride(const int64_t *st, const int64_t *n, int dims, int head_dim, int esize)
{
    for (int i = 0; i < dims; ++i) {
        if (n[i] < 2) continue;                           // never stepped over
        if (st[i] < head_dim || st[i] >= ((int64_t)1 << 40) / esize || st[i] * esize % 16 != 0) return OBF_ERR_INVALID_ARG;
    }
    return OBF_OK;
}

static obf_status_t validate_attend(const obf_attend_t *a, const obf_prefix_t *x)
{
    if (!a) return OBF_ERR_INVALID_ARG;
    if (a->batch < 1 || a->kv_heads < 1 || a->q_heads < 1 || a->q_heads % a->kv_heads != 0) return OBF_ERR_INVALID_ARG;
    if (a->n_q < 1 || a->n_q > OBF_MAX_T || a->capacity < 1 || a->capacity > OBF_MAX_T) return OBF_ERR_INVALID_ARG;
    if (a->window < 0 || a->sinks < 0) return OBF_ERR_INVALID_ARG;
    if (!(a->scale >= 0.f) || !std::isfinite(a->scale) || !(a->decay >= 0.f) || !std::isfinite(a->decay)) return OBF_ERR_INVALID_ARG;
    if (a->flags & ~(uint32_t)(OBF_FLAG_GENERIC_PATH | OBF_FLAG_TEST_WAIT_EXPIRES)) return OBF_ERR_INVALID_ARG;
    if (a->head_dim != 64 && a->head_dim != 128) return OBF_ERR_UNSUPPORTED;
    if (a->dtype != OBF_F32 && a->dtype != OBF_BF16) return OBF_ERR_UNSUPPORTED;
    if ((long long)a->batch * a->q_heads > (1 << 24) || (long long)a->batch * a->q_heads * a->n_q > 1ll << 30) return OBF_ERR_UNSUPPORTED;
    if (x) {
        if (x->rows < 1 || x->rows > OBF_MAX_T) return OBF_ERR_INVALID_ARG;
        if (a->window || a->sinks || a->mass_in || a->mass_out) return OBF_ERR_INVALID_ARG;
    }
    if (a->mass_in && !a->mass_out) return OBF_ERR_INVALID_ARG;
    if (a->mass_out && (long long)(a->q_heads / a->kv_heads) * a->n_q > 64) return OBF_ERR_UNSUPPORTED;
    return OBF_OK;
}

static obf_status_t validate_attend_pointers(const obf_attend_t *a, const obf_prefix_t *x)
{
    const int es = a->dtype == OBF_F32 ? 4 : 2;
    if (!a->q || !a->k || !a->v || !a->out || misaligned(a->q) || misaligned(a->k) || misaligned(a->v) || misaligned(a->out)) return OBF_ERR_INVALID_ARG;
    const int64_t nq[3] = {a->batch, a->q_heads, a->n_q}, nk[3] = {a->batch, a->kv_heads, a->capacity};
    OBF_TRY(check_stride(a->q_stride, nq, 3, a->head_dim, es));
    OBF_TRY(check_stride(a->out_stride, nq, 3, a->head_dim, es));
    OBF_TRY(check_stride(a->k_stride, nk, 3, a->head_dim, es));
    OBF_TRY(check_stride(a->v_stride, nk, 3, a->head_dim, es));
    if (x) {
        if (!x->k || !x->v || misaligned(x->k) || misaligned(x->v)) return OBF_ERR_INVALID_ARG;
        const int64_t np[2] = {a->kv_heads, x->rows};
        OBF_TRY(check_stride(x->k_stride, np, 2, a->head_dim, es));
        OBF_TRY(check_stride(x->v_stride, np, 2, a->head_dim, es));
    }
    const void *words[] = {a->lens, a->q_lens, a->lse_out, a->mass_in, a->mass_out};
    for (const void *w : words)
        if (reinterpret_cast<uintptr_t>(w) & 3u) return OBF_ERR_INVALID_ARG;
    return OBF_OK;
}

// Kernels that a set of keys (a sequence's own ones, the shared prefix) is worked on by.
enum AttendPath { ATTEND_GENERIC, ATTEND_FEW, ATTEND_TC };

struct AttendLayout {
    AttendPath own_path, p_path;
    int p_slots, own_slots;          // parts of the prefix and of a sequence's own keys
    bool cluster;                    // the parts join themselves
    bool with_prefix;                // and walk the prefix as well
    size_t off_part_o, off_part_lse, off_logits, total;
};

// Parts of `keys` keys for `tiles` tiles of query rows: about `blocks` blocks in all, at least `least` keys each.
static int parts_for(long long tiles, long long keys, long long blocks, int least)
{
    long long s = (blocks + tiles - 1) / tiles, most = (keys + least - 1) / least;
    if (s > most) s = most;
    if (s > 128) s = 128;
    return (int)(s < 1 ? 1 : s);
}

// Keys that a query row can see at most.
static long long most_keys(const obf_attend_t *a, int rows_of_queries)
{
    if (a->window == 0) return a->capacity;
    const long long n = (long long)a->window + rows_of_queries + a->sinks;
    return n < a->capacity ? n : a->capacity;
}

// Up to 16 query rows (and a mass call's at most 64) go where a tile of 128 rows, or the generic kernel's 64, would stay empty.
static AttendPath path_for(const obf_attend_t *a, long long rows)
{
    if (a->flags & OBF_FLAG_GENERIC_PATH) return ATTEND_GENERIC;
    if (rows <= 16 || a->mass_out) return ATTEND_FEW;
    if (a->dtype != OBF_BF16) return ATTEND_GENERIC;
    return a->q_heads / a->kv_heads <= AT_TILE ? ATTEND_TC : ATTEND_GENERIC;
}

constexpr int FEW_RESIDENT = 2 * 148;        // blocks of k_attend_few that run at once; of k_attend_few_f32 twice as many

// Query rows of a tile of the kernels for few rows.
static int few_rows(int dtype, long long rows) { return dtype == OBF_F32 ? (rows <= 4 ? 4 : 8) : rows <= 8 ? 8 : 16; }

// Tiles of query rows on the tensor cores: `ti` queries of `nb` sequences with the G heads of the group.
struct TcTiles {
    int ti, nb;
    long long pairs;                 // pairs of tiles over the call
};

static TcTiles tc_tiles(int G, int n_q, int batch, int kv_heads, bool prefix)
{
    TcTiles t;
    t.ti = AT_TILE / G < n_q ? AT_TILE / G : n_q;
    t.nb = 1;
    t.pairs = (long long)kv_heads * batch * ((n_q + 2 * t.ti - 1) / (2 * t.ti));
    if (!prefix) return t;
    // 8 sequences of 40 queries x 4 heads: 10 full tiles of 8 queries of 4 sequences, not 16 of a sequence's 32 or 8 queries
    long long fewest = LLONG_MAX;
    for (int ti = t.ti; ti >= 1; --ti) {
        const int nb = AT_TILE / (G * ti) < batch ? AT_TILE / (G * ti) : batch;
        const long long tiles = (long long)((n_q + ti - 1) / ti) * ((batch + nb - 1) / nb);
        if (tiles < fewest) { fewest = tiles; t.ti = ti; t.nb = nb; }
    }
    t.pairs = kv_heads * ((fewest + 1) / 2);
    return t;
}

// Parts of the keys for the persistent kernel: as many as make its last round of items (one per multiprocessor) fullest,
// counting an item's fixed cost as that of one tile of keys, a join where there would be none (no other keys: `joined` false) as
// two tiles, and a pair's partial results on their way there as a hundredth.  (32 heads over 8, on the device: prompt of 512 alone
// 15.4 us in 1 part, 23.1 in 2; 4 x 64 queries over 600 keys 17.9 in 1, 19.7 in 3; 256 queries over 2048 keys 24.5 in 4.)
static int tc_parts(long long pairs, long long keys, bool joined)
{
    const long long tiles = (keys + AT_TILE - 1) / AT_TILE;
    int best = 1;
    double cost = 1e300;
    for (int s = 1; s <= 128 && s <= (tiles + 1) / 2; ++s) {
        const double c = (double)((pairs * s + 147) / 148) * ((double)((tiles + s - 1) / s) + 1.0 + (s > 1 ? 0.5 : 0.0)) +
                         (s > 1 && !joined ? 2.0 : 0.0) + (s > 1 || joined ? 0.01 * (double)(s * pairs) : 0.0);
        if (c < cost * 0.97) { cost = c; best = s; }
        if (pairs * s > 148 * 4) break;
    }
    return best;
}

// Parts of the keys for k_attend_few: as many as make its rounds of resident blocks cheapest, a block costing its keys and, to
// begin and to end, as much as 120 more; at least 256 keys each.  (Measured beside one another: 16 sequences of 8192
// keys and their masses, 128 tiles: the rule's 9 parts 96 us, 18 parts 99, 28 parts 101; 32 of up to 8192 with a window of 4096: the rule's
// 1 part 74.6, 9 parts 80; 4 of 131072: the rule's 37 parts 283, 9 parts 286, 18 parts 281, 28 parts, whose last round is the emptiest, 292.)
static int few_parts(long long tiles, long long keys, int resident)
{
    long long best = 1, cost = LLONG_MAX;
    for (long long s = 1; s <= 128 && (s == 1 || s * 256 <= keys); ++s) {
        const long long c = (tiles * s + resident - 1) / resident * ((keys + s - 1) / s + 120);
        if (c < cost) { cost = c; best = s; }
    }
    return (int)best;
}

// Whether the call may ask for waits that run out: small ones that the tensor-core kernel works on.
static bool may_expire(const obf_attend_t *a, const obf_prefix_t *x)
{
    const long long rows = (long long)(a->q_heads / a->kv_heads) * a->n_q;
    return !x && path_for(a, rows) == ATTEND_TC && (long long)a->batch * a->kv_heads <= 4 && a->n_q <= 2048 && a->capacity <= 2048;
}

static AttendLayout attend_layout(const obf_attend_t *a, const obf_prefix_t *x)
{
    AttendLayout L;
    const long long rows_seq = (long long)(a->q_heads / a->kv_heads) * a->n_q, heads = (long long)a->batch * a->kv_heads, rows = heads * rows_seq;
    const auto parts = [&](AttendPath path, long long runs, long long rows_run, long long keys) {
        if (path == ATTEND_FEW) {
            // small calls: short parts, up to eight of them, a cluster each
            const int t = few_rows(a->dtype, rows_run);
            const long long tiles = runs * ((rows_run + t - 1) / t);
            if (8 * tiles <= FEW_RESIDENT && keys <= 4096) return parts_for(1, keys, 8, 64);
            return few_parts(tiles, keys, a->dtype == OBF_F32 ? 2 * FEW_RESIDENT : FEW_RESIDENT);
        }
        if (path == ATTEND_TC) return tc_parts(tc_tiles((int)(a->q_heads / a->kv_heads), a->n_q, a->batch, a->kv_heads, rows_run != rows_seq).pairs, keys, x != nullptr);
        return parts_for(runs * ((rows_run + AG_TILE - 1) / AG_TILE), keys, 2 * 148, 4 * AG_TILE);
    };
    L.own_path = path_for(a, rows_seq);
    L.own_slots = parts(L.own_path, heads, rows_seq, most_keys(a, AG_TILE));
    L.p_path = ATTEND_GENERIC;
    L.p_slots = 0;
    // A small call over a prefix: three launches would take longer than reading it once per sequence, from the L2 cache, as long as
    // the clusters all run at once.  (us from Python, one launch and three, measured beside one another; 8 KV heads, relay of 1012 rows:
    // 4 sequences 14.7 and 19.1; 5, whose 320 blocks do not fit, 17.2 and 19.7, replayed from a graph 16.3 and 13.6; 16: 34.9 and 19.7.  Of
    // 256 rows 5 sequences 12.0 and 19.9, 32: 28.6 and 19.6.  4 sequences, 4000 rows: 15.8 and 19.1, from a graph 15.0 and 14.8; 4200:
    // 17.2 and 19.7, 16.3 and 13.6; 12000: 35.4 and 20.2.)
    const long long few_tiles = heads * ((rows_seq + few_rows(a->dtype, rows_seq) - 1) / few_rows(a->dtype, rows_seq));
    L.with_prefix = x && L.own_path == ATTEND_FEW && 8 * few_tiles <= FEW_RESIDENT && x->rows + a->capacity <= 4096;
    if (L.with_prefix) {
        L.own_slots = parts_for(1, x->rows + a->capacity, 8, 64);
    } else if (x) {
        L.p_path = path_for(a, a->batch * rows_seq);
        L.p_slots = parts(L.p_path, a->kv_heads, a->batch * rows_seq, x->rows);
    }
    const int slots = L.own_slots + L.p_slots;
    size_t o = 256;
    // Parts that all fit the chip at once join themselves (replayed from a graph, without and with a join's launch: a token over 1024 keys
    // 6.7 us and 6.7, with a window of 256 5.2 and 6.1, four sequences 7.6 and 8.0; over 4096 keys the join is the better
    // there, 12.8 and 10.9); more of them wait for places for whole clusters, which costs more than the join (batch of
    // 32, 1024 blocks: 81 us instead of 77).
    // (masses: the blocks of a cluster have to see all rows of the head)
    L.cluster = L.with_prefix || (L.own_path == ATTEND_FEW && !x && (a->mass_out ? rows_seq <= few_rows(a->dtype, rows_seq) : slots > 1) && slots <= 8 &&
                                  few_tiles * slots <= FEW_RESIDENT);
    const bool join = (slots > 1 || a->mass_out) && !L.cluster;
    L.off_part_o = o;
    if (join) o = align_up(o + (size_t)slots * rows * a->head_dim * sizeof(float), 256);
    L.off_part_lse = o;
    if (join) o = align_up(o + (size_t)slots * rows * sizeof(float), 256);
    L.off_logits = o;
    if (a->mass_out) o = align_up(o + (size_t)rows * a->capacity * sizeof(float), 256);
    L.total = o;
    return L;
}

// Raises a kernel's shared-memory limit the first time it is used on a device.
template <typename K>
static obf_status_t set_smem_once(K kernel, size_t bytes, bool (&done)[64])
{
    int dev = 0;
    OBF_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 0 && dev < 64 && done[dev]) return OBF_OK;
    OBF_TRY(set_smem(kernel, bytes));
    if (dev >= 0 && dev < 64) done[dev] = true;
    return OBF_OK;
}

template <typename TIN, int D, bool PREFIX>
static obf_status_t launch_attend_generic(const AttendDev &p, int first, cudaStream_t st)
{
    static bool done[64];
    OBF_TRY(set_smem_once(k_attend_generic<TIN, D, PREFIX>, attend_generic_smem<TIN, D>(), done));
    const long long rows = (PREFIX ? (long long)p.batch : 1) * p.n_q * p.G, tiles = (rows + AG_TILE - 1) / AG_TILE;
    const long long blocks = (PREFIX ? p.p_slots : p.slots - p.p_slots) * tiles * p.kv_heads * (PREFIX ? 1 : p.batch);
    if (blocks > INT_MAX) return OBF_ERR_UNSUPPORTED;
    OBF_TRY(launch(k_attend_generic<TIN, D, PREFIX>, dim3((unsigned)blocks), AG_NT, attend_generic_smem<TIN, D>(), st, p, first));
    ++g_last_launches;
    return OBF_OK;
}

template <int ROWS, bool PREFIX, bool CLUSTER, typename K>
static obf_status_t launch_few(K kernel, size_t smem, const AttendDev &p, int first, cudaStream_t st)
{
    const int parts = PREFIX ? p.p_slots : p.slots - p.p_slots;
    const long long rows = (PREFIX ? (long long)p.batch : 1) * p.n_q * p.G, tiles = (rows + ROWS - 1) / ROWS;
    const long long blocks = parts * tiles * p.kv_heads * (PREFIX ? 1 : p.batch);
    if (blocks > INT_MAX) return OBF_ERR_UNSUPPORTED;
    OBF_TRY(launch_clusters(CLUSTER ? parts : 1, kernel, dim3((unsigned)blocks), AF_NT, smem, st, p, first));
    ++g_last_launches;
    return OBF_OK;
}

template <typename TIN, int D, int ROWS, bool PREFIX, bool CLUSTER>
static obf_status_t launch_attend_few_rows(const AttendDev &p, int first, cudaStream_t st)
{
    if constexpr (sizeof(TIN) == 4) {
        return launch_few<ROWS, PREFIX, CLUSTER>(k_attend_few_f32<D, ROWS, PREFIX, CLUSTER>, 0, p, first, st);
    } else {
        static bool done[64];
        OBF_TRY(set_smem_once(k_attend_few<D, ROWS / 8, PREFIX, CLUSTER>, attend_few_smem<D>(), done));
        return launch_few<ROWS, PREFIX, CLUSTER>(k_attend_few<D, ROWS / 8, PREFIX, CLUSTER>, attend_few_smem<D>(), p, first, st);
    }
}

template <typename TIN, int D, bool PREFIX>
static obf_status_t launch_attend_few(const AttendDev &p, int first, cudaStream_t st)
{
    constexpr int SMALL = sizeof(TIN) == 4 ? 4 : 8;
    const long long rows = (PREFIX ? (long long)p.batch : 1) * p.n_q * p.G;
    const bool small = few_rows(sizeof(TIN) == 4 ? OBF_F32 : OBF_BF16, rows) == SMALL;
    if constexpr (!PREFIX)
        if (p.cluster) return small ? launch_attend_few_rows<TIN, D, SMALL, false, true>(p, first, st) : launch_attend_few_rows<TIN, D, 2 * SMALL, false, true>(p, first, st);
    return small ? launch_attend_few_rows<TIN, D, SMALL, PREFIX, false>(p, first, st) : launch_attend_few_rows<TIN, D, 2 * SMALL, PREFIX, false>(p, first, st);
}

// Strides of dimensions that are never stepped over may be anything for the caller, not for a tensor map.
static cuuint64_t map_stride(long long elements, uint64_t n) { return n > 1 ? (cuuint64_t)elements * 2 : 16; }

static obf_status_t encode_map(CUtensorMap *m, const void *ptr, int rank, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box)
{
    EncodeTiledFn enc = tensor_map_encoder();
    if (!enc) return OBF_ERR_CUDA;
    const cuuint32_t es[5] = {1, 1, 1, 1, 1};
    const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void *>(ptr), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        std::fprintf(stderr, "obf: cuTensorMapEncodeTiled failed with %d\n", (int)r);
        return OBF_ERR_CUDA;
    }
    return OBF_OK;
}

template <int D, bool PREFIX>
static obf_status_t launch_attend_tc(const AttendDev &p, int first, cudaStream_t st)
{
    static bool done[64];
    // Dynamic shared memory begins behind the 1024 bytes that the system keeps and what the kernel declares; the tiles want
    // multiples of 1024.
    static const size_t smem = [] {
        cudaFuncAttributes fa = {};
        if (cudaFuncGetAttributes(&fa, k_attend_tc<D, PREFIX>) != cudaSuccess) { (void)cudaGetLastError(); return (size_t)0; }
        return align_up(fa.sharedSizeBytes, 1024) - fa.sharedSizeBytes + AttendTcShape<D>::SMEM_BYTES;
    }();
    if (smem == 0) return OBF_ERR_CUDA;
    OBF_TRY(set_smem_once(k_attend_tc<D, PREFIX>, smem, done));
    const TcTiles t = tc_tiles(p.G, p.n_q, p.batch, p.kv_heads, PREFIX);
    AttendTcMaps m;
    m.ti = t.ti;
    m.nb = t.nb;
    const cuuint64_t hq = (cuuint64_t)p.kv_heads * p.G, nq = p.n_q, nb = p.batch, kv = p.kv_heads;
    {
        const cuuint64_t dims[4] = {D, hq, nq, nb}, strides[3] = {map_stride(p.qs[1], hq), map_stride(p.qs[2], nq), map_stride(p.qs[0], nb)};
        const cuuint32_t box[4] = {64, (cuuint32_t)p.G, (cuuint32_t)t.ti, (cuuint32_t)t.nb};
        OBF_TRY(encode_map(&m.q, p.q, 4, dims, strides, box));
    }
    // the sinks take 16, 32, 48 or 64 rows at the front of the first tile of keys, more than that tiles of their own
    m.head_rows = !PREFIX && p.window && p.sinks ? (p.sinks <= 64 ? (p.sinks + 15) / 16 * 16 : (p.sinks + AT_TILE - 1) / AT_TILE * AT_TILE) : 0;
    for (int i = 0; i < 2; ++i) {
        const long long *s3 = i ? p.vs : p.ks, *s2 = i ? p.pvs : p.pks;
        const void *ptr = PREFIX ? (i ? p.pv : p.pk) : (i ? p.v : p.k);
        const cuuint64_t rows = PREFIX ? p.prefix : p.capacity, n = PREFIX ? 1 : nb;
        cuuint64_t dims[5] = {64, rows, D / 64, kv, n};
        const cuuint64_t strides[4] = {map_stride(PREFIX ? s2[1] : s3[2], rows), 128, map_stride(PREFIX ? s2[0] : s3[1], kv), PREFIX ? 16 : map_stride(s3[0], n)};
        cuuint32_t box[5] = {64, AT_TILE, D / 64, 1, 1};
        OBF_TRY(encode_map(i ? &m.v : &m.k, ptr, 5, dims, strides, box));
        if (m.head_rows == 0) continue;
        const bool shared_tile = m.head_rows < AT_TILE;
        if (shared_tile) {
            box[1] = AT_TILE - m.head_rows;
            box[2] = 1;
            OBF_TRY(encode_map(&m.rest[i], ptr, 5, dims, strides, box));
            box[1] = m.head_rows;
        }
        dims[1] = (cuuint64_t)p.sinks < rows ? p.sinks : rows;           // rows behind the sinks read as zero
        OBF_TRY(encode_map(&m.head[i], ptr, 5, dims, strides, box));
    }
    const long long items = t.pairs * (PREFIX ? p.p_slots : p.slots - p.p_slots);
    if (items > INT_MAX / 2) return OBF_ERR_UNSUPPORTED;
    const int blocks = items < sm_count() ? (int)items : sm_count();
    OBF_TRY(launch(k_attend_tc<D, PREFIX>, dim3(blocks), AT_THREADS, smem, st, p, m, (int)items, first));
    ++g_last_launches;
    return OBF_OK;
}

template <typename TIN, int D, bool PREFIX>
static obf_status_t launch_attend(AttendPath path, const AttendDev &p, int first, cudaStream_t st)
{
    if (path == ATTEND_FEW) return launch_attend_few<TIN, D, PREFIX>(p, first, st);
    if constexpr (sizeof(TIN) == 2) {
        if (path == ATTEND_TC) return launch_attend_tc<D, PREFIX>(p, first, st);
    }
    return launch_attend_generic<TIN, D, PREFIX>(p, first, st);
}

template <typename TIN, int D>
static obf_status_t run_attend(const AttendLayout &L, const AttendDev &p, cudaStream_t st)
{
    if (p.prefix) OBF_TRY((launch_attend<TIN, D, true>(L.p_path, p, 1, st)));
    OBF_TRY((launch_attend<TIN, D, false>(L.own_path, p, p.prefix == 0, st)));
    if ((p.slots > 1 || p.mass_out) && !p.cluster) {
        // a warp per row fills the chip from some thousand rows on; fewer are joined by four warps each
        const bool many = p.rows_total >= 4 * 148;
        const long long row_blocks = many ? (p.rows_total + 3) / 4 : p.rows_total;
        long long blocks = row_blocks;
        if (p.mass_out) blocks += (long long)p.batch * p.kv_heads * ((p.capacity + AJ_KEYS - 1) / AJ_KEYS);
        if (blocks > INT_MAX) return OBF_ERR_UNSUPPORTED;
        if (many) OBF_TRY(launch(k_attend_join<TIN, D, 1>, dim3((unsigned)blocks), AJ_NT, 0, st, p, (int)row_blocks));
        else OBF_TRY(launch(k_attend_join<TIN, D, 4>, dim3((unsigned)blocks), AJ_NT, 0, st, p, (int)row_blocks));
        ++g_last_launches;
    }
    return OBF_OK;
}

static obf_status_t attend(const obf_attend_t *a, const obf_prefix_t *x, void *workspace, size_t bytes, void *stream)
{
    g_last_launches = 0;
    OBF_TRY(validate_attend(a, x));
    OBF_TRY(validate_attend_pointers(a, x));
    if ((a->flags & OBF_FLAG_TEST_WAIT_EXPIRES) && !may_expire(a, x)) return OBF_ERR_INVALID_ARG;
    const AttendLayout L = attend_layout(a, x);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || bytes < L.total) return OBF_ERR_WORKSPACE;
    AttendDev p = {};
    p.q = a->q; p.k = a->k; p.v = a->v; p.out = a->out;
    for (int i = 0; i < 3; ++i) { p.qs[i] = a->q_stride[i]; p.ks[i] = a->k_stride[i]; p.vs[i] = a->v_stride[i]; p.os[i] = a->out_stride[i]; }
    if (x) {
        p.pk = x->k; p.pv = x->v;
        (L.with_prefix ? p.with_prefix : p.prefix) = x->rows;
        for (int i = 0; i < 2; ++i) { p.pks[i] = x->k_stride[i]; p.pvs[i] = x->v_stride[i]; }
    }
    p.lens = a->lens; p.q_lens = a->q_lens; p.lse_out = a->lse_out; p.mass_in = a->mass_in; p.mass_out = a->mass_out;
    p.decay = a->decay;
    p.wait_limit_ns = tc::WAIT_LIMIT_NS;
    if (a->flags & OBF_FLAG_TEST_WAIT_EXPIRES) {
        p.wait_limit_ns = 20000000ull;
        p.debug_drop_load = 1;
    }
    p.c = (a->scale > 0.f ? a->scale : 1.f / std::sqrt((float)a->head_dim)) * 1.4426950408889634f;
    p.batch = a->batch; p.kv_heads = a->kv_heads; p.G = a->q_heads / a->kv_heads; p.n_q = a->n_q; p.capacity = a->capacity;
    // beyond any position a window or a number of first tokens changes nothing; clamped, positions minus windows cannot overflow
    p.window = a->window < 2 * OBF_MAX_T ? a->window : 2 * OBF_MAX_T;
    p.sinks = a->sinks < 2 * OBF_MAX_T ? a->sinks : 2 * OBF_MAX_T;
    p.cluster = L.cluster;
    p.p_slots = L.p_slots; p.slots = L.p_slots + L.own_slots;
    p.rows_total = (long long)p.batch * p.kv_heads * p.n_q * p.G;
    char *ws = static_cast<char *>(workspace);
    p.status = reinterpret_cast<uint32_t *>(ws);
    p.part_o = reinterpret_cast<float *>(ws + L.off_part_o);
    p.part_lse = reinterpret_cast<float *>(ws + L.off_part_lse);
    p.logits = reinterpret_cast<float *>(ws + L.off_logits);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->dtype == OBF_F32) return a->head_dim == 64 ? run_attend<float, 64>(L, p, st) : run_attend<float, 128>(L, p, st);
    return a->head_dim == 64 ? run_attend<__nv_bfloat16, 64>(L, p, st) : run_attend<__nv_bfloat16, 128>(L, p, st);
}

template <int ROW_BYTES>
static obf_status_t launch_evict(const EvictDev &p, cudaStream_t st)
{
    const long long heads = (long long)p.batch * p.kv_heads;
    if (p.capacity > EM_CACHE) {
        const long long blocks = heads * ((p.keep + EC_ROWS - 1) / EC_ROWS);
        if (blocks > INT_MAX) return OBF_ERR_UNSUPPORTED;
        OBF_TRY(launch(k_evict_select, dim3((unsigned)heads), ES_NT, 0, st, p));
        OBF_TRY(launch(k_evict_copy<ROW_BYTES>, dim3((unsigned)blocks), EM_NT, 0, st, p));
        g_last_launches += 2;
        return OBF_OK;
    }
    const dim3 grid((unsigned)(heads * p.parts));
    if (p.capacity <= 4 * EM_NT) OBF_TRY(launch(k_evict_mass<ROW_BYTES, 4>, grid, EM_NT, 0, st, p));
    else if (p.capacity <= 16 * EM_NT) OBF_TRY(launch(k_evict_mass<ROW_BYTES, 16>, grid, EM_NT, 0, st, p));
    else OBF_TRY(launch(k_evict_mass<ROW_BYTES, 32>, grid, EM_NT, 0, st, p));
    ++g_last_launches;
    return OBF_OK;
}

}  // namespace obf

using namespace obf;

extern "C" {

obf_status_t obf_attend_workspace_bytes(const obf_attend_t *args, const obf_prefix_t *prefix, size_t *bytes)
{
    if (!bytes) return OBF_ERR_INVALID_ARG;
    OBF_TRY(validate_attend(args, prefix));
    if ((args->flags & OBF_FLAG_TEST_WAIT_EXPIRES) && !may_expire(args, prefix)) return OBF_ERR_INVALID_ARG;
    *bytes = attend_layout(args, prefix).total;
    return OBF_OK;
}

obf_status_t obf_attend(const obf_attend_t *args, void *workspace, size_t workspace_bytes, void *stream)
{
    return attend(args, nullptr, workspace, workspace_bytes, stream);
}

obf_status_t obf_attend_shared(const obf_attend_t *args, const obf_prefix_t *prefix, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!prefix) return OBF_ERR_INVALID_ARG;
    return attend(args, prefix, workspace, workspace_bytes, stream);
}

obf_status_t obf_evict_by_mass(const obf_evict_t *a, void *stream)
{
    g_last_launches = 0;
    if (!a) return OBF_ERR_INVALID_ARG;
    if (a->batch < 1 || a->kv_heads < 1 || a->capacity < 1 || a->capacity > OBF_MAX_T) return OBF_ERR_INVALID_ARG;
    if (a->keep < 1 || a->keep > OBF_MAX_T || a->sinks < 0 || a->recent < 0 || (long long)a->sinks + a->recent > a->keep) return OBF_ERR_INVALID_ARG;
    if (a->head_dim != 64 && a->head_dim != 128) return OBF_ERR_UNSUPPORTED;
    if (a->dtype != OBF_F32 && a->dtype != OBF_BF16) return OBF_ERR_UNSUPPORTED;
    const long long heads = (long long)a->batch * a->kv_heads;
    if (heads > 1 << 24) return OBF_ERR_UNSUPPORTED;
    if (!a->k || !a->v || !a->k_out || !a->v_out || !a->mass || !a->idx_out || misaligned(a->k) || misaligned(a->v) || misaligned(a->k_out) || misaligned(a->v_out))
        return OBF_ERR_INVALID_ARG;
    const void *words[] = {a->mass, a->lens, a->idx_out, a->mass_out, a->lens_out};
    for (const void *w : words)
        if (reinterpret_cast<uintptr_t>(w) & 3u) return OBF_ERR_INVALID_ARG;
    if (a->mass_out && a->mass_out_rows < a->keep) return OBF_ERR_INVALID_ARG;
    const int es = a->dtype == OBF_F32 ? 4 : 2;
    const int64_t ni[3] = {a->batch, a->kv_heads, a->capacity}, no[3] = {a->batch, a->kv_heads, a->keep};
    OBF_TRY(check_stride(a->k_stride, ni, 3, a->head_dim, es));
    OBF_TRY(check_stride(a->v_stride, ni, 3, a->head_dim, es));
    OBF_TRY(check_stride(a->k_out_stride, no, 3, a->head_dim, es));
    OBF_TRY(check_stride(a->v_out_stride, no, 3, a->head_dim, es));
    EvictDev p = {};
    p.k = a->k; p.v = a->v; p.k_out = a->k_out; p.v_out = a->v_out;
    for (int i = 0; i < 3; ++i) { p.ks[i] = a->k_stride[i] * es; p.vs[i] = a->v_stride[i] * es; p.kos[i] = a->k_out_stride[i] * es; p.vos[i] = a->v_out_stride[i] * es; }
    p.mass = a->mass; p.lens = a->lens; p.idx_out = a->idx_out; p.mass_out = a->mass_out; p.lens_out = a->lens_out;
    p.batch = a->batch; p.kv_heads = a->kv_heads; p.capacity = a->capacity; p.keep = a->keep; p.sinks = a->sinks; p.recent = a->recent;
    p.mass_out_rows = a->mass_out_rows;
    // as many blocks as run at once, two per multiprocessor, at least 64 rows each
    const int kept = a->keep < a->capacity ? a->keep : a->capacity;
    long long parts = 2 * 148 / heads;
    if (parts > (kept + 63) / 64) parts = (kept + 63) / 64;
    p.parts = parts < 1 ? 1 : (int)parts;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (a->head_dim * es) {
    case 128: return launch_evict<128>(p, st);
    case 256: return launch_evict<256>(p, st);
    default: return launch_evict<512>(p, st);
    }
}

}  // extern "C"
