/*
 * obf.h - C ABI of the relay-boundary prompt-KV compressor for NVIDIA B200 (sm_100a).
 *
 * One call compresses the prompt KV cache of one or more agents at the relay
 * boundary.  For every (cache, layer, KV head), independently (Section 4.4):
 *
 *   a1  score    A_j = sum over the observation queries t mapped to this KV head of
 *                softmax_j(q_t . K_j / sqrt(head_dim))            (Eq. 1; softmax form of App. L.1)
 *   a2  select   the k_eff = min(budget, T) positions of largest A_j, equal masses
 *                resolved towards the lower position, emitted in ascending
 *                position order                                   (Section 4.3.2; Section 3.1)
 *   a3  gather   K_keep = K[idx,:], V_keep = V[idx,:]             (Algorithm 2, last step)
 *   a4  OBF      orthonormal basis of span(V_keep) (Eq. 2); residual of the deleted
 *                values against that span (Eq. 3); its top-`rank` right singular
 *                subspace C; attention-weighted residual mean r_bar (Eq. 4);
 *                Delta = (r_bar C^T) C (Eq. 5); delta = A_del/(A_keep+eps) * Delta
 *                (Eq. 6); V_out = V_keep + delta on every retained row, keys
 *                untouched (Eq. 7; Algorithm 3)
 *
 * All pointers in obf_cache_t are DEVICE pointers unless a function says
 * otherwise.  The caller owns every buffer, including the workspace; the
 * library allocates no device memory, enqueues all work on `stream`, never
 * synchronises (except obf_last_device_status and the *_host entry point's
 * final wait, as documented) and does not touch the inputs after the enqueued
 * work has completed.  Inputs are read-only and must not alias outputs.
 *
 * Layout (row-major, contiguous, 16-byte aligned base pointers):
 *   k, v      [layers, kv_heads, T, head_dim]
 *   q_obs     [layers, q_heads, n_obs, head_dim]   q head = kv_head * G + g, G = q_heads / kv_heads
 *   k_out,
 *   v_out     [layers, kv_heads, k_eff, head_dim]  same dtype as the inputs
 *   idx_out   [layers, kv_heads, k_eff] int32      ascending positions in [0, T)
 *
 * Numerics: bf16 products accumulated in fp32; softmax, pooling, selection
 * keys and all OBF algebra in fp32; V_out is the fp32 sum rounded once to the
 * output dtype (bit-exact copy of V_keep wherever delta == 0).  K_out is always
 * a bit-exact copy.
 *
 * Errors: anything detectable on the host (null or misaligned pointer, bad
 * shape, budget < 1, rank outside [0, head_dim], unsupported head_dim or dtype,
 * workspace too small) returns a code before anything is enqueued.  Conditions
 * only the device can see are ORed into a status word in the workspace (and
 * into obf_diag_t.status of the head concerned); obf_last_device_status reads
 * it.  A head that hits one keeps its eviction-only result (the skip rule in
 * the footnote to Eq. 7).
 */
#ifndef OBF_H_
#define OBF_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    OBF_OK = 0,
    OBF_ERR_INVALID_ARG = 1,    /* null/misaligned pointer, bad shape, budget, rank, n_caches    */
    OBF_ERR_UNSUPPORTED = 2,    /* head_dim not in {64,128}, unknown dtype, too many caches       */
    OBF_ERR_WORKSPACE = 3,      /* workspace null, misaligned or smaller than obf_workspace_bytes */
    OBF_ERR_CUDA = 4,           /* a CUDA runtime call failed (launch, attribute, copy)           */
    OBF_ERR_DEVICE_STATUS = 5   /* the device status word is non-zero (obf_last_device_status)    */
} obf_status_t;

typedef enum { OBF_F32 = 0, OBF_BF16 = 1 } obf_dtype_t;

/* Bits of the device status word / obf_diag_t.status. */
#define OBF_DEV_NONFINITE   0x1u   /* a score or softmax normaliser was not finite                 */
#define OBF_DEV_NO_CONVERGE 0x2u   /* the eigen-iteration hit its sweep limit                      */
#define OBF_DEV_TIMEOUT     0x4u   /* a bounded on-device wait expired                             */
#define OBF_DEV_INTERNAL    0x8u   /* an internal consistency check failed (position out of range) */
#define OBF_DEV_SKIPPED     0x100u /* informational (diag only): OBF skipped, delta = 0            */
#define OBF_DEV_SPAN_FULL   0x200u /* informational (diag only): span(V_keep) is all of R^d        */

/* obf_params_t.flags */
#define OBF_FLAG_GENERIC_PATH 0x1u /* run the shape-generic kernels even where the tuned bf16 path applies */
#define OBF_FLAG_LAYERWISE    0x2u /* layerwise selector (Section 3.2 retention rule, second form; Algorithm 2,
                                      granularity L): the retained positions of a layer are TopK_B of the masses
                                      summed over its KV heads and are shared by those heads (idx_out repeats them
                                      per head); gather and OBF then run per head with the head's own masses.
                                      Needs every T <= 16384, else OBF_ERR_UNSUPPORTED                          */

#define OBF_FLAG_FAST_PATH    0x4u /* the principal subspace of the residual comes from three steps of the Gram
                                      subspace iteration of App. H, C <- orth(C R^T R), started at the first rows of
                                      the identity (the paper leaves the start open), instead of the exact
                                      eigenvectors: an approximation whose error depends on the residual's spectrum.
                                      diag: lam_1 / lam_rho are Rayleigh quotients, lam_next is 0                  */
#define OBF_FLAG_ATTN_INJECT  0x8u /* Attn-inject (App. D.2, alternative designs): the vector delta of Eq. 6 is added in
                                      proportion to each retained position's attention mass instead of uniformly,
                                      V*_t = V_t + k_eff * A_t / (A_keep + eps) * delta (the shares average one).
                                      delta_out and the diagnostics are those of the uniform injection             */
#define OBF_FLAG_MERGE        0x10u /* cache-merging baseline instead of Orthogonal BackFill (App. E, the comparison
                                      method): after selection and gather every deleted position is routed to the
                                      retained position with the most similar key (cosine; ties: lowest position) and
                                      V*_t = V_t + sum over the j routed to t of A_j / (A_t + eps) V_j.  params->rank is
                                      ignored; delta_out stays zero                                                */
#define OBF_FLAG_EARLY_OUT    0x20u /* the span test before the pass over V (tuned bf16 path, rank > 0): a head whose
                                      retained values span R^d has delta = 0 whatever its deleted values are (Eq. 3),
                                      so that pass skips it.  Same outputs bit for bit; the call's kernels then run
                                      one after the other on `stream` instead of beside one another.  Pays when most
                                      heads have budgets of head_dim or more; without the flag every head's values
                                      are streamed                                                                 */
#define OBF_FLAG_SINK(n) (((uint32_t)(n) & 0xFFu) << 8)
                                   /* protected sink prefix (App. F of the paper: the compressors protect the first s
                                      indices of the cache; the eligible set of Section 3.2 leaves the sink out): the
                                      first n <= 255 positions of every cache are retained besides the budget and are no
                                      candidates of the selection, so k_eff = min(n, T) + min(budget, T - min(n, T));
                                      size the outputs with that k_eff                                            */
#define OBF_FLAG_SINK_OF(flags) (((flags) >> 8) & 0xFFu)
#define OBF_FLAG_TEST_WAIT_EXPIRES 0x10000u
                                   /* test hook for the bounded device-side waits of the tuned score kernel: no block
                                      publishes a head's softmax normalisers and the wait limit drops from one second to
                                      20 ms, so every wait for them runs out, the kernels return by themselves, the
                                      status word carries OBF_DEV_TIMEOUT and the outputs hold valid positions but no
                                      meaningful selection.  Accepted only for at most 4 (layer, KV head) pairs in all,
                                      every T <= 2048, on the tuned bf16 path; else
                                      OBF_ERR_INVALID_ARG.  In obf_attend, for that of the tensor-core kernel: no block
                                      fetches the values of its first tile of keys, out and lse hold anything; for
                                      batch * kv_heads <= 4 and n_q, capacity <= 2048, where that kernel is used  */

#define OBF_MAX_CACHES 32          /* caches per call                                              */
#define OBF_MAX_T (1 << 20)        /* prompt positions per cache                                   */

typedef struct {              /* shared by all caches of one call                                   */
    int32_t layers, kv_heads, q_heads;  /* q_heads % kv_heads == 0                                  */
    int32_t head_dim;                   /* 64 or 128                                                */
    int32_t n_obs;                      /* observation queries per query head (>= 1)                */
    int32_t rank;                       /* pca_rank of Section 4.4; 0 = eviction only               */
    int32_t dtype;                      /* obf_dtype_t of k, v, q_obs, k_out, v_out                 */
    float   eps;                        /* the epsilon of Eq. 4 and Eq. 6 (the paper uses 1e-12)    */
    uint32_t flags;                     /* OBF_FLAG_*                                               */
} obf_params_t;

typedef struct {              /* per (layer, KV head) diagnostics (App. K.2 names in brackets)      */
    float a_keep, a_del;      /* attention mass on retained / deleted positions (Eq. 6)             */
    float alpha;              /* a_del / (a_keep + eps)                              [DR]           */
    float rcr;                /* ||R||_F^2 / (||V_del||_F^2 + eps)                   [RCR]          */
    float delta_norm;         /* ||delta||_2                                         [IVN]          */
    float kth_score;          /* smallest retained mass among the candidates of the selection       */
    float next_score;         /* largest deleted mass, -1 if nothing is deleted                     */
    float lam_1, lam_rho, lam_next; /* eigenvalues of R^T R: largest, last kept, first dropped      */
    int32_t span_rank;        /* numerical dimension m of span(V_keep) (-1: not evaluated)          */
    int32_t rho_eff;          /* number of principal directions actually used                       */
    uint32_t status;          /* OBF_DEV_* bits                                                     */
    float revr;               /* sum of the rho_eff kept eigenvalues of R^T R over their total  [REVR]; PCR is 1 - rcr */
    float pc;                 /* cosine between the sum of the deleted values and the sum of their projections onto
                                 span(V_keep)  [PC]; 0 when OBF does not run for the head; costs one more pass over V,
                                 made only when diag_out is given                                        */
} obf_diag_t;

typedef struct {              /* one agent's prompt cache; T and budget may differ between caches   */
    const void *k, *v;        /* [layers, kv_heads, T, head_dim]                                    */
    const void *q_obs;        /* [layers, q_heads, n_obs, head_dim]                                 */
    int32_t T;                /* prompt positions, 1 <= T <= OBF_MAX_T                              */
    int32_t budget;           /* >= 1; k_eff = min(budget, T) (more with OBF_FLAG_SINK, see there)  */
    void *k_out, *v_out;      /* [layers, kv_heads, k_eff, head_dim]                                */
    int32_t *idx_out;         /* [layers, kv_heads, k_eff]                                          */
    obf_diag_t *diag_out;     /* optional [layers, kv_heads], or NULL                               */
    float *scores_out;        /* optional [layers, kv_heads, T] attention mass A (Eq. 1), or NULL   */
    float *delta_out;         /* optional [layers, kv_heads, head_dim] injected vector (Eq. 6), or NULL */
    const float *lse_extra;   /* optional device [layers, q_heads, n_obs] fp32, or NULL: per observation query the
                                 natural log of the sum of exp(q.k / sqrt(d)) over the keys OUTSIDE the prompt that the
                                 model's softmax also ran over (earlier agents' relay, the latent positions before it:
                                 Section 3.1 defines the weights of Eq. 1 as a softmax over the whole cache, App. L.1
                                 restates it over the prompt).  Those keys take their share of every row's
                                 normaliser, so a row's weights over the prompt add up to less than one.  NULL or
                                 minus infinity: softmax over the prompt keys alone                          */
    /* Optional int8 copy of the compacted relay (post-hoc quantisation stacked on the compression, App. E, Table 7;
       the paper fixes no quantiser: symmetric, one fp32 scale per retained row, scale = max|x| / 127, code =
       round-half-even(x / scale), a row of zeros has scale 0).  All four NULL, or all four device pointers:
       k_q8_out, v_q8_out int8 [layers, kv_heads, k_eff, head_dim]; k_scale_out, v_scale_out fp32
       [layers, kv_heads, k_eff]; the int8 arrays 8-byte aligned, the scales 4-byte aligned.  The codes are taken
       from k_out / v_out as the call leaves them (v_out after the injection of Eq. 7), which are still written. */
    int8_t *k_q8_out, *v_q8_out;
    float *k_scale_out, *v_scale_out;
    int32_t *assign_out;      /* optional device [layers, kv_heads, T], or NULL; with OBF_FLAG_MERGE: the slot
                                 (0 .. k_eff-1) every deleted position was routed to, -1 for retained positions   */
} obf_cache_t;

/*
 * Size in bytes of the scratch workspace obf_compress / evict_only need for
 * this call shape (Eq. 1's masses, selection flags, the d x d Gram matrices of
 * Eq. 3 and App. H).  Host-only; enqueues nothing.  Pointers inside `caches`
 * are not inspected, only T and budget.
 */
obf_status_t obf_workspace_bytes(const obf_params_t *params, const obf_cache_t *caches,
                                 int32_t n_caches, size_t *bytes);

/*
 * Phi_OBF (Algorithm 3) on every (cache, layer, KV head).  `params`/`caches`
 * are host structs (copied before return); `workspace` is device memory of at
 * least obf_workspace_bytes(), 256-byte aligned, private to this call until
 * the enqueued work completes; `stream` is a cudaStream_t passed as void*.
 * With rank > 0 on the tuned path the selection, the gather of the values and
 * the span test run on a stream of the library (created on first use per host
 * thread and device) that forks from and joins `stream` inside the call,
 * beside the pass over V (heads of 64 channels: without the selection, which
 * that pass waits for): everything the call does is ordered on `stream`.
 *
 * Calls that overlap on one device (different streams or host threads, each
 * with its own workspace) are legal but do not speed each other up: the tuned
 * score kernel's blocks wait for one another, so it is launched cooperatively
 * and starts only when the whole grid (one block per multiprocessor) can be
 * resident; until then it waits for whatever else holds the multiprocessors.
 * Every device-side wait is bounded (one second): if one ever runs out the
 * kernels return by themselves, the status word carries OBF_DEV_TIMEOUT (see
 * obf_last_device_status) and the outputs hold valid positions but no
 * meaningful selection.
 */
obf_status_t obf_compress(const obf_params_t *params, const obf_cache_t *caches, int32_t n_caches,
                          void *workspace, size_t workspace_bytes, void *stream);

/*
 * Phi_Attn with headwise granularity (Algorithm 2): steps a1-a3 only.
 * Identical to obf_compress with rank = 0 (params->rank is ignored).
 */
obf_status_t evict_only(const obf_params_t *params, const obf_cache_t *caches, int32_t n_caches,
                        void *workspace, size_t workspace_bytes, void *stream);

/*
 * Size of the device arena obf_compress_host needs (device copies of every
 * input and output of the call plus the workspace).
 */
obf_status_t obf_host_arena_bytes(const obf_params_t *params, const obf_cache_t *caches,
                                  int32_t n_caches, size_t *bytes);

/*
 * Same operation for callers whose caches live in HOST memory (Algorithm 1's
 * relay hand-off when the cache is staged on the host).  Every pointer inside
 * `caches` is a host pointer (pinned memory makes the copies asynchronous);
 * `device_arena` is device memory of at least obf_host_arena_bytes(),
 * 256-byte aligned.  Copies k, v, q_obs to the device, compresses, and copies
 * k_out, v_out, idx_out (and the optional outputs that are not NULL) back,
 * as a pipeline over slabs of layers: the copies run on two streams that
 * the library creates on first use (per host thread and device), the
 * kernels on `stream`; work already enqueued on `stream` is waited for
 * first.  Returns after everything has finished.  The injected vectors can
 * differ from obf_compress on the same data in the last fp32 digits (a slab
 * adds its partial sums up in another order than the whole call).
 */
obf_status_t obf_compress_host(const obf_params_t *params, const obf_cache_t *caches, int32_t n_caches,
                               void *device_arena, size_t arena_bytes, void *stream);

/*
 * Waits for `stream`, reads the status word the last call left in `workspace`
 * and stores it in *device_status.  Returns OBF_ERR_DEVICE_STATUS if any of
 * the error bits (OBF_DEV_NONFINITE, OBF_DEV_NO_CONVERGE, OBF_DEV_TIMEOUT,
 * OBF_DEV_INTERNAL) is set.
 */
obf_status_t obf_last_device_status(const void *workspace, void *stream, uint32_t *device_status);

/*
 * obf_compress with per-kernel device timing, for profiling only.  Enqueues the
 * same kernels as obf_compress (params->rank == 0 gives evict_only's), with a
 * CUDA event recorded between consecutive launches, waits for the stream and
 * writes the elapsed milliseconds of each launch to phase_ms[0 .. *n_phases-1]
 * (host array with room for OBF_MAX_PHASES floats).  obf_phase_name(i) names
 * launch i of the last profiled call of this thread.
 */
#define OBF_MAX_PHASES 16
obf_status_t obf_compress_profiled(const obf_params_t *params, const obf_cache_t *caches, int32_t n_caches,
                                   void *workspace, size_t workspace_bytes, void *stream,
                                   float *phase_ms, int32_t *n_phases);
const char *obf_phase_name(int32_t phase);

/*
 * evict_only for callers that cannot obtain a workspace.  (The paper has no
 * counterpart: this entry point exists for deployment reasons only.)
 *
 * Some hosts of this library cannot call cudaMalloc at the point where they
 * need a compression: a serving process whose start-up code handed every byte
 * of device memory to its own pool, a plug-in that runs under another
 * framework's allocator and must not allocate behind its back, or a latency
 * critical loop that cannot take the device-wide synchronisation an allocation
 * implies.  For them the scratch memory lives inside the library: a fixed
 * array of OBF_STATIC_SCRATCH_BYTES bytes in the library's device image, which
 * every GPU that loads the library holds until the process exits.  The caller
 * passes only inputs and outputs (all device pointers, as for evict_only).
 *
 * - Computes exactly what evict_only computes (steps a1-a3; params->rank is
 *   ignored) and returns the same codes, plus OBF_ERR_WORKSPACE - with a
 *   message on stderr naming both sizes - when the call shape needs more
 *   scratch than OBF_STATIC_SCRATCH_BYTES (obf_workspace_bytes with rank 0
 *   tells how much a shape needs; for bf16 heads of 64 channels the size with
 *   OBF_FLAG_GENERIC_PATH, less its key splits, decides, for bf16 heads of 128
 *   channels that with the tensor-core kernel's statistics, 1 KB a head and 128
 *   query rows, per 512 positions instead of 256: a call that only those
 *   statistics make too large is enqueued as groups of
 *   heads, or of layers with OBF_FLAG_LAYERWISE, one after the other.  Where
 *   not even one such head or layer of every cache fits, the shape-generic
 *   kernels run, whose masses differ in the last fp32 digits).
 * - Calls no cudaMalloc, cudaFree or any other allocating routine.
 * - The first call on each device resolves the array's device address
 *   (cudaGetSymbolAddress, with that device current); make that first call
 *   before starting any stream capture on the device.  Host threads may make
 *   their first calls at the same time (the address is kept in an atomic).
 * - All calls on one device share the one array and it keeps whatever the
 *   previous call left; the call clears the part that has to start at zero
 *   (the status word) and overwrites the rest before reading it.  Two calls
 *   whose work overlaps on the GPU (different streams, or different host
 *   threads) race on the array: serialise them.
 * - obf_static_scratch_status reads the status word of the last such call.
 */
#define OBF_STATIC_SCRATCH_BYTES (8u << 20)
obf_status_t evict_only_static(const obf_params_t *params, const obf_cache_t *caches, int32_t n_caches,
                               void *stream);
obf_status_t obf_static_scratch_status(void *stream, uint32_t *device_status);

/* ------------------------------------------------------------------------------------------------------------------
 * Operators on a relayed cache: what a user does with the cache after the hand-off.  (The paper relays through its host
 * framework's attention; these entry points are the library's own.)
 *
 * The next agent attends over the relayed cache and appends to it (obf_attend), several agents read one relay
 * (obf_attend_shared), and a cache that has grown is brought down again by the attention mass that its positions have
 * received since (obf_evict_by_mass).  One call is one layer of a batch of sequences: keys and values
 * [batch, kv_heads, capacity, head_dim], queries [batch, q_heads, n_q, head_dim], q head = kv_head * G + g.  Lengths are
 * read on the device, so a captured call can be replayed while the caches grow.
 * ---------------------------------------------------------------------------------------------------------------- */

/*
 * Attention of n_q queries per sequence and query head over a cache.  Sequence b holds lens[b] keys (rows 0 .. lens[b] - 1)
 * and q_lens[b] queries; query i is the token at position t = lens[b] - q_lens[b] + i and sees key j <= t when
 *
 *     window == 0   or   j > t - window   or   j < sinks
 *
 * (a sliding window, its own position included, and the first tokens, which stay visible).  With x_j = scale q . k_j over
 * the visible keys:  out = sum_j softmax_j(x) v_j,  lse = ln sum_j exp(x_j),  and, when mass_out is given, for every KV head
 * and key j < lens[b]
 *
 *     mass_out_j = decay * mass_in_j + sum over the head's G q_lens[b] query rows of softmax_j(x)          (Eq. 1, kept up
 *                                                                                                    while decoding)
 *
 * A query that sees no key (t < 0, when q_lens[b] > lens[b]) has out = 0 and lse = -infinity.  What lies behind a
 * length - queries and outputs from q_lens[b] on, keys, values and masses from lens[b] on - is not read into any result
 * and left as it was; so are values that no query of the sequence sees, whatever they hold.  (A value that is not finite
 * and that some query sees may also spoil queries of the same head that do not see it, as 0 * inf does in a matrix product.)
 * lens outside [0, capacity] and q_lens outside [0, n_q] are clamped and set OBF_DEV_INTERNAL in the status word.
 * obf_cache_t.lse_extra of a later compression is the lse of its observation queries over the keys outside the prompt.
 *
 * Numerics: products of the inputs accumulated in fp32, softmax in fp32; on the tensor cores the weights of a row, at most
 * one, are rounded to bf16 before they multiply the values (their sum is not), out is rounded once.  Weights are kept
 * relative to a reference that may be off a row's maximum by factors of up to 2^32 or 2^-47: values beyond 2^90, or beyond
 * 2^100 divided by the number of keys that a query sees, may overflow in sums that would not, and of values below 2^-60
 * precision may be lost.  A sequence's result does not depend
 * on what else the batch holds except through the batch's sizes - over a shared prefix, where rows of several sequences
 * are worked on together, only in its rounding - and is the same in every run.
 */
typedef struct {
    int32_t batch, kv_heads, q_heads;   /* q_heads % kv_heads == 0                                               */
    int32_t head_dim;                   /* 64 or 128                                                             */
    int32_t n_q;                        /* query rows per sequence and query head, 1 <= n_q <= OBF_MAX_T         */
    int32_t capacity;                   /* rows of k and v per sequence and KV head, 1 <= capacity <= OBF_MAX_T  */
    int32_t window;                     /* >= 0; 0: every key up to the query's own                              */
    int32_t sinks;                      /* >= 0; has no effect without a window                                  */
    int32_t dtype;                      /* obf_dtype_t of q, k, v, out                                           */
    float scale;                        /* factor of the logits, > 0; 0: 1 / sqrt(head_dim)                      */
    float decay;                        /* >= 0; factor of mass_in                                               */
    uint32_t flags;                     /* 0, OBF_FLAG_GENERIC_PATH (CUDA-core kernels where the tensor cores apply) or
                                           OBF_FLAG_TEST_WAIT_EXPIRES                                            */
    const void *q, *k, *v;              /* device, 16-byte aligned                                               */
    void *out;                          /* [batch, q_heads, n_q, head_dim], must not overlap the inputs          */
    int64_t q_stride[3], k_stride[3], v_stride[3], out_stride[3];
                                        /* elements from one sequence, head and row to the next; channels are
                                           contiguous.  Multiples of 16 bytes, at least head_dim and less than 2^40
                                           bytes where there is more than one of them, in any order ([batch, n_q, q_heads, head_dim] is one)   */
    const int32_t *lens;                /* device [batch], or NULL: capacity                                     */
    const int32_t *q_lens;              /* device [batch], or NULL: n_q                                          */
    float *lse_out;                     /* device [batch, q_heads, n_q], or NULL                                 */
    const float *mass_in;               /* device [batch, kv_heads, capacity], or NULL: zeros                    */
    float *mass_out;                    /* the same, or NULL; may be mass_in.  Needs G * n_q <= 64, else
                                           OBF_ERR_UNSUPPORTED (a prompt's masses are obf_compress's scores_out)  */
} obf_attend_t;

/* Keys and values that every sequence of a batch sees before its own. */
typedef struct {
    const void *k, *v;                  /* device, 16-byte aligned, [kv_heads, rows, head_dim]                   */
    int64_t k_stride[2], v_stride[2];   /* elements from one head and row to the next, as above                  */
    int32_t rows;                       /* 1 <= rows <= OBF_MAX_T                                                */
} obf_prefix_t;

/* Device scratch for obf_attend (prefix NULL) or obf_attend_shared.  Host-only; pointers are not inspected, but whether
   mass_out is NULL counts. */
obf_status_t obf_attend_workspace_bytes(const obf_attend_t *args, const obf_prefix_t *prefix, size_t *bytes);

/*
 * Enqueues the attention on `stream`; allocates nothing and never synchronises, can be captured into a graph.  `workspace`:
 * at least obf_attend_workspace_bytes(), 256-byte aligned, private to the call until its work is done (two captured graphs
 * that share one must not overlap); nothing in it is kept from call to call except the status word that
 * obf_last_device_status reads.  Device-side waits are bounded, as in obf_compress.  The first call of a kind on a device raises its
 * kernels' shared-memory limits: make it before a stream capture.
 */
obf_status_t obf_attend(const obf_attend_t *args, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The same over a prefix that all sequences share and each sequence's own keys behind it: every query sees all rows of the
 * prefix and the keys of its own sequence up to its own position (t counts own keys; with t < 0 the prefix alone).  The
 * prefix is read from memory once for the queries of all sequences together.  window, sinks, mass_in and mass_out must be 0 / NULL.
 */
obf_status_t obf_attend_shared(const obf_attend_t *args, const obf_prefix_t *prefix, void *workspace, size_t workspace_bytes,
                               void *stream);

/*
 * Eviction by accumulated mass: of the lens[b] rows of every (sequence, KV head) the first `sinks`, the last `recent` and,
 * of the others, those of largest mass are kept, min(keep, lens[b]) in all; equal masses are resolved towards the lower
 * position, a mass that is not a number counts as the lowest.  Kept rows are copied in ascending order to rows
 * 0 .. min(keep, lens[b]) - 1 of the outputs; what lies behind them is left as it was.  With lens[b] <= keep every row is
 * kept.  Inputs must not overlap outputs.  lens outside [0, capacity] are clamped.
 */
typedef struct {
    int32_t batch, kv_heads, head_dim, capacity, dtype;   /* as above                                            */
    int32_t keep;                       /* 1 <= keep <= OBF_MAX_T, keep >= sinks + recent                        */
    int32_t sinks, recent;              /* >= 0                                                                  */
    const void *k, *v;
    void *k_out, *v_out;                /* [batch, kv_heads, >= keep, head_dim]                                  */
    int64_t k_stride[3], v_stride[3], k_out_stride[3], v_out_stride[3];
    const float *mass;                  /* device [batch, kv_heads, capacity]                                    */
    const int32_t *lens;                /* device [batch], or NULL: capacity                                     */
    int32_t *idx_out;                   /* device [batch, kv_heads, keep] kept positions                         */
    float *mass_out;                    /* device [batch, kv_heads, mass_out_rows] masses of the kept rows, or NULL */
    int32_t mass_out_rows;              /* >= keep (the capacity of the cache that the outputs go on as)         */
    int32_t *lens_out;                  /* device [batch], or NULL: min(keep, lens[b])                           */
} obf_evict_t;

/* Enqueues the eviction on `stream`; needs no workspace, allocates nothing and never synchronises. */
obf_status_t obf_evict_by_mass(const obf_evict_t *args, void *stream);

/* Static, never NULL. */
const char *obf_status_string(obf_status_t status);

/* Number of kernels the last call of this thread that enqueues work enqueued. */
int32_t obf_last_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* OBF_H_ */
