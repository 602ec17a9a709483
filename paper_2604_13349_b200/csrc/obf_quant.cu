// Host side of a relayed cache held in 8 or 4 bits (include/obf.h): argument validation, workspace layout, kernel dispatch.
#include <cmath>

#include "attend_host.cuh"
#include "attend_quant.cuh"
#include "attend_quant_few.cuh"
#include "host.cuh"
#include "quant_cache.cuh"

namespace obf {

static bool quant_strides(const int64_t *st, const int64_t *n, int64_t row, int64_t most)
{
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (st[i] < row || st[i] >= most || st[i] % row != 0)) return false;
    return true;
}

static obf_status_t validate_cache(const obf_quantized_t *c, int batch, int kv_heads, int head_dim, int capacity)
{
    if (!c) return OBF_ERR_INVALID_ARG;
    if (batch < 1 || kv_heads < 1 || capacity < 1 || capacity > OBF_MAX_T) return OBF_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return OBF_ERR_UNSUPPORTED;
    if (c->bits != 8 && c->bits != 4) return OBF_ERR_UNSUPPORTED;
    if ((long long)batch * kv_heads > 1 << 24) return OBF_ERR_UNSUPPORTED;
    return OBF_OK;
}

static obf_status_t validate_cache_pointers(const obf_quantized_t *c, int batch, int kv_heads, int head_dim, int capacity)
{
    if (!c->k || !c->v || !c->k_scale || !c->v_scale || misaligned(c->k) || misaligned(c->v)) return OBF_ERR_INVALID_ARG;
    const int64_t n[3] = {batch, kv_heads, capacity}, row = head_dim * c->bits / 8, per = c->bits == 8 ? 1 : head_dim / 32, es = c->bits == 8 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale)) & (per * es - 1)) return OBF_ERR_INVALID_ARG;
    for (const int64_t *st : {c->k_stride, c->v_stride})
        for (int i = 0; i < 3; ++i)
            if (n[i] > 1 && (st[i] < row || st[i] >= (int64_t)1 << 40 || st[i] % 16 != 0)) return OBF_ERR_INVALID_ARG;
    const int64_t most = ((int64_t)1 << 40) / es;
    if (!quant_strides(c->k_scale_stride, n, per, most) || !quant_strides(c->v_scale_stride, n, per, most)) return OBF_ERR_INVALID_ARG;
    return OBF_OK;
}

static QuantDev quant_dev(const obf_quantized_t *c)
{
    const int es = c->bits == 8 ? 4 : 2;
    QuantDev d;
    d.k = static_cast<const uint8_t *>(c->k);
    d.v = static_cast<const uint8_t *>(c->v);
    d.k_scale = static_cast<const uint8_t *>(c->k_scale);
    d.v_scale = static_cast<const uint8_t *>(c->v_scale);
    for (int i = 0; i < 3; ++i) {
        d.ks[i] = c->k_stride[i]; d.vs[i] = c->v_stride[i];
        d.kss[i] = c->k_scale_stride[i] * es; d.vss[i] = c->v_scale_stride[i] * es;
    }
    return d;
}

// Runs body with the call's type, bits and channels as constants.
template <typename F>
static obf_status_t with_shape(int dtype, int bits, int head_dim, F body)
{
    const auto bits_dim = [&](auto t) {
        typedef decltype(t) T;
        if (bits == 4) return head_dim == 64 ? body(T(), std::integral_constant<int, 4>(), std::integral_constant<int, 64>())
                                             : body(T(), std::integral_constant<int, 4>(), std::integral_constant<int, 128>());
        return head_dim == 64 ? body(T(), std::integral_constant<int, 8>(), std::integral_constant<int, 64>())
                              : body(T(), std::integral_constant<int, 8>(), std::integral_constant<int, 128>());
    };
    return dtype == OBF_F32 ? bits_dim(float()) : bits_dim(__nv_bfloat16());
}

// The rows of a call to write or read, `per` a block; UNSUPPORTED where they cannot be numbered in 31 bits.
static obf_status_t rows_dev(RowsDev *p, int batch, int kv_heads, int rows, int first, int capacity, const int32_t *lens, unsigned *blocks, int per)
{
    const long long half = (long long)batch * kv_heads * rows;
    if (2 * half > INT_MAX - per) return OBF_ERR_UNSUPPORTED;
    p->lens = lens;
    p->rows = rows; p->first = first; p->capacity = capacity;
    p->half = (uint32_t)half; p->total = (uint32_t)(2 * half);
    p->by_rows = fast_div(rows);
    p->by_heads = fast_div(kv_heads);
    *blocks = (unsigned)((2 * half + per - 1) / per);
    return OBF_OK;
}

static obf_status_t validate_words(const void *a, const void *b)
{
    return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & 3u) ? OBF_ERR_INVALID_ARG : OBF_OK;
}

static obf_status_t quant_write(const obf_quantized_write_t *a, const obf_quantized_t *c, cudaStream_t st)
{
    g_last_launches = 0;
    if (!a) return OBF_ERR_INVALID_ARG;
    OBF_TRY(validate_cache(c, a->batch, a->kv_heads, a->head_dim, a->capacity));
    if (a->rows < 1 || a->rows > OBF_MAX_T) return OBF_ERR_INVALID_ARG;
    if (a->dtype != OBF_F32 && a->dtype != OBF_BF16) return OBF_ERR_UNSUPPORTED;
    OBF_TRY(validate_cache_pointers(c, a->batch, a->kv_heads, a->head_dim, a->capacity));
    if (!a->k || !a->v || misaligned(a->k) || misaligned(a->v) || !a->k_values != !a->v_values || misaligned(a->k_values) || misaligned(a->v_values))
        return OBF_ERR_INVALID_ARG;
    const int es = a->dtype == OBF_F32 ? 4 : 2;
    const int64_t n[3] = {a->batch, a->kv_heads, a->rows};
    OBF_TRY(check_stride(a->k_stride, n, 3, a->head_dim, es));
    OBF_TRY(check_stride(a->v_stride, n, 3, a->head_dim, es));
    if (a->k_values) {
        OBF_TRY(check_stride(a->k_values_stride, n, 3, a->head_dim, es));
        OBF_TRY(check_stride(a->v_values_stride, n, 3, a->head_dim, es));
    }
    OBF_TRY(validate_words(a->lens, a->new_lens));
    RowsDev p = {};
    unsigned blocks;
    const int ahead = a->dtype == OBF_BF16 ? (c->bits == 4 ? QW_AHEAD<__nv_bfloat16, 4> : QW_AHEAD<__nv_bfloat16, 8>)
                                           : (c->bits == 4 ? QW_AHEAD<float, 4> : QW_AHEAD<float, 8>);
    OBF_TRY(rows_dev(&p, a->batch, a->kv_heads, a->rows, 0, a->capacity, a->lens, &blocks, QC_NT / (a->head_dim / 16) * ahead));
    p.new_lens = a->new_lens;
    p.k = a->k; p.v = a->v; p.k_out = a->k_values; p.v_out = a->v_values;
    for (int i = 0; i < 3; ++i) { p.ks[i] = a->k_stride[i]; p.vs[i] = a->v_stride[i]; p.kos[i] = a->k_values_stride[i]; p.vos[i] = a->v_values_stride[i]; }
    const QuantDev d = quant_dev(c);
    return with_shape(a->dtype, c->bits, a->head_dim, [&](auto t, auto bits, auto dim) -> obf_status_t {
        typedef decltype(t) T;
        if (p.k_out) OBF_TRY(launch(k_quant_write<T, bits.value, dim.value, true>, dim3(blocks), QC_NT, 0, st, p, d));
        else OBF_TRY(launch(k_quant_write<T, bits.value, dim.value, false>, dim3(blocks), QC_NT, 0, st, p, d));
        ++g_last_launches;
        return OBF_OK;
    });
}

static obf_status_t quant_read(const obf_quantized_read_t *a, const obf_quantized_t *c, cudaStream_t st)
{
    g_last_launches = 0;
    if (!a) return OBF_ERR_INVALID_ARG;
    OBF_TRY(validate_cache(c, a->batch, a->kv_heads, a->head_dim, a->capacity));
    if (a->first < 0 || a->rows < 1 || (long long)a->first + a->rows > a->capacity) return OBF_ERR_INVALID_ARG;
    if (a->dtype != OBF_F32 && a->dtype != OBF_BF16) return OBF_ERR_UNSUPPORTED;
    OBF_TRY(validate_cache_pointers(c, a->batch, a->kv_heads, a->head_dim, a->capacity));
    if (!a->k_out || !a->v_out || misaligned(a->k_out) || misaligned(a->v_out)) return OBF_ERR_INVALID_ARG;
    const int es = a->dtype == OBF_F32 ? 4 : 2;
    const int64_t n[3] = {a->batch, a->kv_heads, a->rows};
    OBF_TRY(check_stride(a->k_out_stride, n, 3, a->head_dim, es));
    OBF_TRY(check_stride(a->v_out_stride, n, 3, a->head_dim, es));
    OBF_TRY(validate_words(a->lens, nullptr));
    RowsDev p = {};
    unsigned blocks;
    OBF_TRY(rows_dev(&p, a->batch, a->kv_heads, a->rows, a->first, a->capacity, a->lens, &blocks, QC_NT / (a->head_dim / 16) * QR_AHEAD));
    p.k_out = a->k_out; p.v_out = a->v_out;
    for (int i = 0; i < 3; ++i) { p.kos[i] = a->k_out_stride[i]; p.vos[i] = a->v_out_stride[i]; }
    const QuantDev d = quant_dev(c);
    return with_shape(a->dtype, c->bits, a->head_dim, [&](auto t, auto bits, auto dim) -> obf_status_t {
        OBF_TRY(launch(k_quant_read<decltype(t), bits.value, dim.value, false>, dim3(blocks), QC_NT, 0, st, p, d));
        ++g_last_launches;
        return OBF_OK;
    });
}

// ---- attention ------------------------------------------------------------------------------------------------

static obf_status_t validate_attend_quant(const obf_attend_t *a, const obf_quantized_t *c)
{
    if (!a) return OBF_ERR_INVALID_ARG;
    if (a->q_heads < 1 || a->kv_heads < 1 || a->q_heads % a->kv_heads != 0) return OBF_ERR_INVALID_ARG;
    OBF_TRY(validate_cache(c, a->batch, a->kv_heads, a->head_dim, a->capacity));
    if (a->n_q < 1 || a->n_q > OBF_MAX_T || a->window < 0 || a->sinks < 0) return OBF_ERR_INVALID_ARG;
    if (!(a->scale >= 0.f) || !std::isfinite(a->scale)) return OBF_ERR_INVALID_ARG;
    if (a->flags & ~(uint32_t)OBF_FLAG_GENERIC_PATH) return OBF_ERR_INVALID_ARG;
    if (a->dtype != OBF_F32 && a->dtype != OBF_BF16) return OBF_ERR_UNSUPPORTED;
    if (a->mass_in || a->mass_out) return OBF_ERR_UNSUPPORTED;
    if ((long long)a->batch * a->q_heads > (1 << 24) || (long long)a->batch * a->q_heads * a->n_q > 1ll << 30) return OBF_ERR_UNSUPPORTED;
    return OBF_OK;
}

struct QuantLayout {
    bool tiles;                      // rows read back first, attention over them in tiles of 128 query rows
    int slots;                       // parts of the keys
    bool cluster;                    // which join themselves
    size_t off_part_o, off_part_lse;
    size_t rows_bytes, off_k, off_v, off_factors;      // tiles: that attention's workspace, the rows, 8 bits: their factors
    long long factor_stride;
    size_t total;
};

// Query rows of a KV head from which on bf16 calls read the cache's rows back and attend over those on the tensor cores' tiles of 128 rows.
// (16 sequences of 7000 to 8192 keys of 128 channels, us, on codes and on rows read back: 4 bits, 64 rows 185 and 223, 96 rows 264 and 225; 8 bits, 96 rows
// 215 and 275, 112 rows 293 and 275.  64 channels: 4 bits, 64 rows 109 and 155; 4 of 4096 keys, 128 rows 36.4 and 34.4; 8 bits, 96 rows 148 and 197, 128 rows 188 and 197.)
static long long quant_tiles_from(int bits, int head_dim) { return bits == 8 ? (head_dim == 128 ? 97 : 129) : head_dim == 128 ? 81 : 113; }
// In small calls the two launches more take longer.  (us on codes and on rows read back: 2 x 40 queries of 32 heads over 1012 keys in 4 bits, 2.6 million rows times
// keys, 22.4 and 23.2, in 8 bits 18.6 and 25.7; 2 x 64 in 8 bits, 4.1 million, 22.2 and 27.0; a prompt of 128, 0.5 million, in 4 bits 8.4 and 13.4, of 512, 8.4 million,
// 36.2 and 20.2, in 8 bits 31.5 and 20.7; 2 x 200, 13 million, 56.1 and 33.3.)
constexpr long long QUANT_TILES_WORK = 6000000;
// What the rows may take of a workspace.
constexpr size_t QUANT_ROWS_BYTES = (size_t)4 << 30;

// Query rows of a tile: 4 and 8 of k_attend_quant_few, 16, 24 and 32 of k_attend_quant: as many as registers hold, in fp32 no more than 24, in 4 bits at 128
// channels more than 16 only where one tile does.  (16 sequences of 7000 to 8192 keys of 128 channels, us: 20 rows in a tile of 24 and in two of 16
// 90 and 111, fp32 145 and 172; 64 rows in tiles of 32 and 16 179 and 190 in 8 bits, 222 and 185 in 4 bits, of 64 channels 109 and 121; fp32 in tiles of 24
// and 16 340 and 308 in 4 bits.)
static int quant_rows(int dtype, int bits, int head_dim, long long rows)
{
    if (rows <= 8) return rows <= 4 ? 4 : 8;
    if (rows <= 24) return rows <= 16 ? 16 : 24;
    return bits == 4 && head_dim == 128 ? 16 : dtype == OBF_F32 ? 24 : 32;
}

// Runs body with a tile's rows as a constant.
template <typename T, int BITS, int D, typename F>
static obf_status_t with_rows(int rows, F body)
{
    if (rows == 4) return body(std::integral_constant<int, 4>());
    if (rows == 8) return body(std::integral_constant<int, 8>());
    if constexpr (sizeof(T) == 4)
        if (rows == 24) return body(std::integral_constant<int, 24>());
    if constexpr (sizeof(T) == 2) {
        if (rows == 24) return body(std::integral_constant<int, 24>());
        if constexpr (BITS == 8 || D == 64)
            if (rows == 32) return body(std::integral_constant<int, 32>());
    }
    return body(std::integral_constant<int, 16>());
}

// Blocks of a multiprocessor.
template <typename T, int BITS, int D, int ROWS>
static constexpr int blocks_of()
{
    if constexpr (ROWS >= 16) return AQ_BLOCKS<T, BITS, D, ROWS / 8>;
    else return AQF_BLOCKS<T, ROWS / 4>;
}

static QuantLayout quant_layout(const obf_attend_t *a, int bits)
{
    QuantLayout L = {};
    const long long rows_seq = (long long)(a->q_heads / a->kv_heads) * a->n_q, heads = (long long)a->batch * a->kv_heads, rows = heads * rows_seq;
    const size_t rows_kv = (size_t)heads * a->capacity * a->head_dim * 2;
    L.tiles = a->dtype == OBF_BF16 && !(a->flags & OBF_FLAG_GENERIC_PATH) && rows_seq >= quant_tiles_from(bits, a->head_dim) &&
              rows * most_keys(a, 128) >= QUANT_TILES_WORK && 2 * rows_kv <= QUANT_ROWS_BYTES && attends_in_tiles(a);
    if (L.tiles) {
        size_t o = L.rows_bytes = align_up(attend_rows_bytes(a), 256);
        L.off_k = o;
        o = align_up(o + rows_kv, 256);
        L.off_v = o;
        o = align_up(o + rows_kv, 256);
        L.off_factors = o;
        if (bits == 8) {
            L.factor_stride = (long long)align_up(a->capacity, 4);
            o = align_up(o + ((size_t)heads * L.factor_stride + 128) * 2 * sizeof(float), 256);
        }
        L.total = o;
        return L;
    }
    const int t = quant_rows(a->dtype, bits, a->head_dim, rows_seq);
    const long long tiles = heads * ((rows_seq + t - 1) / t), keys = most_keys(a, t);
    int resident = 0;                                     // blocks that run at once
    (void)with_shape(a->dtype, bits, a->head_dim, [&](auto tin, auto nbits, auto dim) -> obf_status_t {
        return with_rows<decltype(tin), nbits.value, dim.value>(t, [&](auto rows) -> obf_status_t {
            resident = 148 * blocks_of<decltype(tin), nbits.value, dim.value, rows.value>();
            return OBF_OK;
        });
    });
    const bool small = 8 * tiles <= resident && keys <= 4096;
    L.slots = small ? parts_for(1, keys, 8, 64) : few_parts(tiles, keys, resident);
    L.cluster = L.slots > 1 && L.slots <= 8 && tiles * L.slots <= resident;
    const bool join = L.slots > 1 && !L.cluster;
    size_t o = 256;
    L.off_part_o = o;
    if (join) o = align_up(o + (size_t)L.slots * rows * a->head_dim * sizeof(float), 256);
    L.off_part_lse = o;
    if (join) o = align_up(o + (size_t)L.slots * rows * sizeof(float), 256);
    L.total = o;
    return L;
}

template <typename T, int BITS, int D, int ROWS, bool CLUSTER>
static obf_status_t launch_quant_rows(const AttendDev &p, const QuantDev &d, cudaStream_t st)
{
    static bool done[64];
    constexpr size_t smem = attend_quant_smem<BITS, D, ROWS>(ROWS >= 16 ? sizeof(QuantQueries<T, BITS, D, ROWS / 8>) : 0);
    const auto kernel = [] {
        if constexpr (ROWS >= 16) return k_attend_quant<T, BITS, D, ROWS / 8, CLUSTER>;
        else return k_attend_quant_few<T, BITS, D, ROWS / 4, CLUSTER>;
    }();
    OBF_TRY(set_smem_once(kernel, smem, done));
    const long long blocks = (long long)p.slots * (((long long)p.n_q * p.G + ROWS - 1) / ROWS) * p.kv_heads * p.batch;
    if (blocks > INT_MAX) return OBF_ERR_UNSUPPORTED;
    OBF_TRY(launch_clusters(CLUSTER ? p.slots : 1, kernel, dim3((unsigned)blocks), AF_NT, smem, st, p, d));
    ++g_last_launches;
    return OBF_OK;
}

template <typename T, int BITS, int D>
static obf_status_t launch_quant(const AttendDev &p, const QuantDev &d, cudaStream_t st)
{
    const auto rows = [&](auto cluster) -> obf_status_t {
        return with_rows<T, BITS, D>(quant_rows(sizeof(T) == 4 ? OBF_F32 : OBF_BF16, BITS, D, (long long)p.n_q * p.G),
                                     [&](auto rows_tile) -> obf_status_t { return launch_quant_rows<T, BITS, D, rows_tile.value, cluster.value>(p, d, st); });
    };
    if (p.cluster) return rows(std::true_type());
    OBF_TRY(rows(std::false_type()));
    if (p.slots > 1) OBF_TRY((launch_join<T, D>(p, st)));
    return OBF_OK;
}

static float logit_factor(const obf_attend_t *a) { return (a->scale > 0.f ? a->scale : 1.f / std::sqrt((float)a->head_dim)) * 1.4426950408889634f; }

// The rows that the queries see are read back, in 4 bits as their values, which are bf16 numbers, in 8 bits as codes, which are too, with their
// scales apart; attention goes over those.
static obf_status_t attend_tiles(const QuantLayout &L, const obf_attend_t *a, const obf_quantized_t *c, char *ws, cudaStream_t st)
{
    RowsDev p = {};
    unsigned blocks;
    OBF_TRY(rows_dev(&p, a->batch, a->kv_heads, a->capacity, 0, a->capacity, a->lens, &blocks, QC_NT / (a->head_dim / 16) * QR_AHEAD));
    obf_attend_t r = *a;
    r.k = p.k_out = ws + L.off_k;
    r.v = p.v_out = ws + L.off_v;
    const int64_t row = a->head_dim, head = row * a->capacity, seq = head * a->kv_heads, stride[3] = {seq, head, row};
    for (int i = 0; i < 3; ++i) p.kos[i] = p.vos[i] = r.k_stride[i] = r.v_stride[i] = stride[i];
    p.q_lens = a->q_lens; p.n_q = a->n_q;
    p.window = a->window < 2 * OBF_MAX_T ? a->window : 2 * OBF_MAX_T;
    p.sinks = a->sinks;
    AttendFactors factors = {};
    if (c->bits == 8) {
        p.factors = reinterpret_cast<float *>(ws + L.off_factors);
        p.factor_stride = L.factor_stride;
        p.c = logit_factor(a);
        factors = {reinterpret_cast<const float4 *>(p.factors), L.factor_stride};
    }
    const QuantDev d = quant_dev(c);
    OBF_TRY(with_shape(OBF_BF16, c->bits, a->head_dim, [&](auto t, auto bits, auto dim) -> obf_status_t {
        if constexpr (sizeof(t) == 2) OBF_TRY(launch(k_quant_read<decltype(t), bits.value, dim.value, bits.value == 8>, dim3(blocks), QC_NT, 0, st, p, d));
        return OBF_OK;
    }));
    OBF_TRY(attend_rows(&r, factors, ws, L.rows_bytes, st));
    ++g_last_launches;
    return OBF_OK;
}

static obf_status_t attend_quant(const obf_attend_t *a, const obf_quantized_t *c, void *workspace, size_t bytes, cudaStream_t st)
{
    g_last_launches = 0;
    OBF_TRY(validate_attend_quant(a, c));
    OBF_TRY(validate_cache_pointers(c, a->batch, a->kv_heads, a->head_dim, a->capacity));
    if (!a->q || !a->out || misaligned(a->q) || misaligned(a->out) || a->k || a->v) return OBF_ERR_INVALID_ARG;
    const int es = a->dtype == OBF_F32 ? 4 : 2;
    const int64_t nq[3] = {a->batch, a->q_heads, a->n_q};
    OBF_TRY(check_stride(a->q_stride, nq, 3, a->head_dim, es));
    OBF_TRY(check_stride(a->out_stride, nq, 3, a->head_dim, es));
    OBF_TRY(validate_words(a->lens, a->q_lens));
    OBF_TRY(validate_words(a->lse_out, nullptr));
    const QuantLayout L = quant_layout(a, c->bits);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || bytes < L.total) return OBF_ERR_WORKSPACE;
    if (L.tiles) return attend_tiles(L, a, c, static_cast<char *>(workspace), st);
    AttendDev p = {};
    p.q = a->q; p.out = a->out;
    for (int i = 0; i < 3; ++i) { p.qs[i] = a->q_stride[i]; p.os[i] = a->out_stride[i]; }
    p.lens = a->lens; p.q_lens = a->q_lens; p.lse_out = a->lse_out;
    p.c = logit_factor(a);
    p.batch = a->batch; p.kv_heads = a->kv_heads; p.G = a->q_heads / a->kv_heads; p.n_q = a->n_q; p.capacity = a->capacity;
    p.window = a->window < 2 * OBF_MAX_T ? a->window : 2 * OBF_MAX_T;
    p.sinks = a->sinks < 2 * OBF_MAX_T ? a->sinks : 2 * OBF_MAX_T;
    p.cluster = L.cluster;
    p.slots = L.slots;
    p.rows_total = (long long)p.batch * p.kv_heads * p.n_q * p.G;
    char *ws = static_cast<char *>(workspace);
    p.status = reinterpret_cast<uint32_t *>(ws);
    p.part_o = reinterpret_cast<float *>(ws + L.off_part_o);
    p.part_lse = reinterpret_cast<float *>(ws + L.off_part_lse);
    const QuantDev d = quant_dev(c);
    return with_shape(a->dtype, c->bits, a->head_dim,
                      [&](auto t, auto bits, auto dim) -> obf_status_t { return launch_quant<decltype(t), bits.value, dim.value>(p, d, st); });
}

}  // namespace obf

using namespace obf;

extern "C" {

obf_status_t obf_quantized_write(const obf_quantized_write_t *args, const obf_quantized_t *cache, void *stream)
{
    return quant_write(args, cache, static_cast<cudaStream_t>(stream));
}

obf_status_t obf_quantized_read(const obf_quantized_read_t *args, const obf_quantized_t *cache, void *stream)
{
    return quant_read(args, cache, static_cast<cudaStream_t>(stream));
}

obf_status_t obf_attend_quantized_workspace_bytes(const obf_attend_t *args, const obf_quantized_t *cache, size_t *bytes)
{
    if (!bytes) return OBF_ERR_INVALID_ARG;
    OBF_TRY(validate_attend_quant(args, cache));
    *bytes = quant_layout(args, cache->bits).total;
    return OBF_OK;
}

obf_status_t obf_attend_quantized(const obf_attend_t *args, const obf_quantized_t *cache, void *workspace, size_t workspace_bytes, void *stream)
{
    return attend_quant(args, cache, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
