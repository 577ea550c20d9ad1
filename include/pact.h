/*
 * pact.h - C ABI of the PACT visual-token reduction library for NVIDIA B200 (sm_100a).
 *
 * The library implements, on one GPU, the per-request reduction step of
 *   "PACT: Pruning and Clustering-Based Token Reduction for Faster Visual Language Models":
 * importance scoring and pruning (EUTI, Algorithm 1), Distance Bounded Density Peak
 * Clustering of the surviving keys (DBDPC, Algorithm 2), reincorporation of pruned tokens
 * that lie close to a centre (Eq. 8-9) and the merge of every cluster into one hidden state
 * that carries its centre's position id (Eq. 10, Algorithm 3).
 *
 * Conventions that hold for every call
 * ------------------------------------
 *  - All data pointers are DEVICE pointers unless a comment says "host".  The caller owns
 *    every buffer, including the workspace; the library never allocates or frees device
 *    memory inside a stage call and never keeps a pointer after the call returns.
 *  - Work is enqueued on `stream` (a cudaStream_t passed as void*) and the call returns
 *    without synchronising.  Counts that depend on the data (q, C, r ...) stay on the device.
 *  - Matrices are row-major; a leading dimension `ld*` is the row stride in ELEMENTS.
 *    Rows must be 16-byte aligned (base pointer and ld * sizeof(element) multiples of 16).
 *  - Element type of H, K, Q is `in` given to pact_create (bf16 or fp32); H_out has type `out`.
 *  - Every call returns a pact_status.  Host-detectable errors (null pointer, bad size or
 *    alignment, workspace too small, parameter out of range) are reported before anything
 *    is launched.  Device-side problems (a bounded wait that ran out) set counters[PACT_CNT_STATUS]
 *    of the image; the library never traps, aborts or throws.
 *  - A context may be used from one host thread and one stream at a time (the replay of a captured call is a use as well: its
 *    workspace is the one that it was captured with).
 *  - Same inputs give bitwise the same outputs, run after run.
 *
 * Readings of the paper that fix the semantics (the paper is silent on them)
 * ------------------------------------------------------------------------
 *  - Softmax in Eq. 2 runs across the visual tokens, separately per head, without 1/sqrt(d_h).
 *  - Query head j reads key head floor(j * n_kvh / n_qh); the mean over heads uses n_qh.
 *  - Percentile(s, lambda): with m = min(floor(lambda*N + 1e-6), N-1) and tau the (m+1)-th
 *    smallest score, a token is important iff s_i >= tau (Eq. 3) - ties at tau are kept.
 *  - The clustering vector of a token is the concatenation of its key heads (width d_k).
 *  - Distances are clamped to [0, 2]; d_ii = 0; a key whose norm vanishes (below about 1e-19)
 *    is at distance 1 from every other key.
 *  - Density ties go to the lower token index; a vector becomes a centre iff its distance to
 *    every earlier centre is strictly greater than d_c; argmin ties go to the lower cluster id.
 *  - Cluster ids number the centres by ascending token index; merged rows are emitted in
 *    that order in place of the visual span; text rows keep their relative place.
 *  - A pruned token rejoins iff its nearest-centre distance is strictly below
 *    (float)alpha * (float)d_c.
 */
#ifndef PACT_H_
#define PACT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pact_ctx pact_ctx; /* opaque; holds shapes and device properties, no device memory */

typedef enum { PACT_BF16 = 0, PACT_F32 = 1 } pact_dtype;

typedef enum {
  PACT_OK = 0,
  PACT_ERR_INVALID_ARG = -1, /* null pointer, bad size, stride or alignment, parameter out of range */
  PACT_ERR_UNSUPPORTED = -2, /* shape, dtype or device the library has no kernel for            */
  PACT_ERR_WORKSPACE = -3,   /* workspace pointer null, misaligned or too small                 */
  PACT_ERR_CUDA = -4,        /* a CUDA runtime call failed (see pact_last_cuda_error)           */
  PACT_ERR_TIMEOUT = -5,     /* value of counters[PACT_CNT_STATUS] when a bounded device wait ran out */
  PACT_ERR_NO_PAGES = -6     /* status of a pact_cache_plan that asked for more pages than are free   */
} pact_status;

/* Slots of the per-image int32 counters array (device memory, 16 entries). */
enum {
  PACT_CNT_N_OUT = 0,     /* rows of H_out / P_out / size_out that are valid                   */
  PACT_CNT_Q = 1,         /* important (surviving) tokens, |S_important|                        */
  PACT_CNT_C = 2,         /* clusters                                                           */
  PACT_CNT_R = 3,         /* pruned tokens that rejoined a cluster                              */
  PACT_CNT_DISCARDED = 4, /* pruned tokens that did not                                         */
  PACT_CNT_SWEEPS = 5,    /* most sweeps over its rows any CTA made in the centre selection, and passes over
                             rows left open after them; depends on timing                         */
  PACT_CNT_BAND_DC = 6,   /* unordered surviving pairs with |d - d_c| <= 1e-6                   */
  PACT_CNT_BAND_ADC = 7,  /* pruned tokens whose nearest-centre distance is within 1e-6 of alpha*d_c */
  PACT_CNT_STATUS = 8,    /* 0, or a negative pact_status raised on the device                  */
  PACT_CNT_M = 9,         /* pruned tokens, |S_unimportant|                                     */
  PACT_N_COUNTERS = 16
};

/* Flags of pact_params.flags (ablations of Sec. 4 of the paper). */
enum {
  PACT_FLAG_CENTER_ONLY = 1u, /* h'_s = h_s: the centre represents its cluster, no averaging     */
  PACT_FLAG_NO_NORM = 2u,     /* Eq. 2 without the hidden-state norm factor                      */
  PACT_FLAG_NORM_ONLY = 4u    /* Eq. 2 without the global-query factor: s_i = |h_i| / N          */
};

/* Hyper-parameters of Algorithm 3. */
typedef struct {
  double lambda;        /* pruning fraction in [0, 1]                                            */
  float d_c;            /* cutoff, cosine distance, in [0, 2]                                    */
  float d_n;            /* density normaliser of Eq. 6, > 0 (the paper uses 2)                   */
  float alpha;          /* reincorporation tolerance of Eq. 8, >= 0 (the paper uses 1.5); 0 = off */
  int32_t n_prune;      /* >= 0: use this m instead of the one derived from lambda               */
  uint32_t flags;       /* PACT_FLAG_*                                                           */
} pact_params;

/* One independent unit: an image or a video clip inside a sequence of n_total tokens. */
typedef struct {
  const void *H;        /* [n_total, d] hidden states at layer L                                 */
  int64_t ldH;
  const void *K_euti;   /* [N, n_kvh*d_h] keys BEFORE rotary embedding, visual rows only         */
  int64_t ldKe;
  const void *Q_euti;   /* [N, n_qh*d_h] queries BEFORE rotary embedding, visual rows only       */
  int64_t ldQ;
  const void *K_clu;    /* [N, n_kvh*d_h] keys AFTER rotary embedding; may alias K_euti          */
  int64_t ldKc;
  const int32_t *P;     /* [n_total] position ids                                                */
  int32_t n_total;      /* tokens in the sequence (text + visual)                                */
  int32_t vis_start;    /* the visual tokens are rows [vis_start, vis_start + N) of H and P      */
  int32_t N;            /* number of visual tokens, >= 1                                         */
  int32_t reserved;
  void *H_out;          /* [n_total, d] capacity; the first counters[N_OUT] rows are valid        */
  int64_t ldHo;
  int32_t *P_out;       /* [n_total] capacity                                                     */
  int32_t *size_out;    /* [n_total] capacity: cluster size (W of Eq. 11); 1 for text rows        */
  int32_t *label;       /* [N] cluster id of every visual token, -1 = discarded; may be NULL      */
  float *score;         /* [N] EUTI scores; may be NULL                                           */
  uint8_t *keep;        /* [N] 1 = important (survived pruning), 0 = pruned; may be NULL          */
  int32_t *counters;    /* [PACT_N_COUNTERS]                                                      */
  float *logw_out;      /* [n_total] capacity: log(size_out), the additive attention bias log W of
                           Eq. 11 for the reduced sequence (0 for text rows); may be NULL           */
} pact_image;

/* ---- context --------------------------------------------------------------------------- */

/* Creates a context for hidden size d, n_qh query heads, n_kvh key heads of width d_h, on the
 * current CUDA device.  Requirements: d_h * n_kvh and d_h * n_qh and d multiples of 8 (bf16) or
 * 4 (fp32); n_qh a multiple of n_kvh, at most 256; d <= 8192; n_qh * (d_h + 32) <= 28928 (the global query in
 * double has to fit an SM's shared memory); `out` is the element type of H_out. */
pact_status pact_create(pact_ctx **ctx, int d, int n_qh, int n_kvh, int d_h, pact_dtype in,
                        pact_dtype out);
pact_status pact_destroy(pact_ctx *ctx);

/* Bytes of device workspace needed for calls with at most max_batch images of at most max_N
 * visual tokens each.  The workspace must be 256-byte aligned.  Its contents need not be
 * preserved between calls and need no initialisation. */
size_t pact_workspace_bytes(const pact_ctx *ctx, int max_batch, int max_N);

const char *pact_status_string(pact_status s);
/* Text of the last CUDA runtime error seen by this context ("" if none). */
const char *pact_last_cuda_error(const pact_ctx *ctx);

/* Bounds of the device-side waits (Algorithm 2's centre selection is resolved in sweeps over two bit masks,
 * and some of the member lists of Eq. 10 are built behind one barrier between CTAs: those of a whole step of up to 1024 tokens per image on keys that the
 * tensor cores do not take, i.e. fp32, or bf16 whose width is no multiple of 64, unless it is small enough for one cluster).  When a bound is reached the
 * kernel stops waiting, writes PACT_ERR_TIMEOUT to counters[PACT_CNT_STATUS] of the image and carries on
 * within bounds; the call itself still returns PACT_OK and the outputs of that image are not valid.
 * The waits of pact_paged_attention for its copies are bounded too; there the status of the call becomes PACT_ERR_TIMEOUT.
 * barrier_polls: polls of the member-list barrier, and of each wait of pact_paged_attention (default: as many as fit into a second);
 * center_sweeps: sweeps of the centre selection (rows that are
 * still open are then decided without waiting, in at most one pass per surviving token; the same happens, with no
 * status, when no row has been removed for 512 sweeps); 0 restores the default (about a million).  Graphs recorded
 * earlier keep the limits they were recorded with. */
pact_status pact_set_wait_limits(pact_ctx *ctx, int barrier_polls, int center_sweeps);

/* ---- instrumentation ---------------------------------------------------------------------- */

/* Number of kernels this context has launched since it was created. */
long long pact_launch_count(const pact_ctx *ctx);
/* With profiling on, pact_reduce records a CUDA event on `stream` after each of its kernels
 * (first parameter block of a call only).  pact_profile_read waits for the last one and writes
 * the duration of each kernel in milliseconds to ms[0..n), returning n (0 if nothing was
 * recorded).  pact_profile_stage_name(i) names the i-th kernel.  A profiled call is launched kernel by
 * kernel whatever the size of its images.  Off by default. */
pact_status pact_profile_enable(pact_ctx *ctx, int on);
int pact_profile_read(pact_ctx *ctx, float *ms /*host*/, int cap);
const char *pact_profile_stage_name(int i);

/* ---- stage calls (one image) ----------------------------------------------------------- */

/* EUTI score, Eq. 1-2 / Algorithm 1 steps 1-2.
 * Reads img->H (visual rows), K_euti, Q_euti; writes score[N] (fp32).  An infinity or a NaN anywhere in
 * Q_euti or K_euti makes every score NaN (also in pact_reduce, where equal scores all survive); with PACT_FLAG_NORM_ONLY
 * neither is read. */
pact_status pact_importance(pact_ctx *ctx, const pact_image *img /*host*/, const pact_params *p /*host*/,
                            float *score, void *ws, size_t ws_bytes, void *stream);

/* Percentile split, Eq. 3-4 / Algorithm 1 step 3.
 * score[N] -> keep[N] (1 = important), kept_idx[q] and pruned_idx[m] in ascending order
 * (capacity N each), counts[0] = q, counts[1] = m (device int32[2]). */
pact_status pact_prune(pact_ctx *ctx, const float *score, int N, const pact_params *p /*host*/,
                       uint8_t *keep, int32_t *kept_idx, int32_t *pruned_idx, int32_t *counts,
                       void *ws, size_t ws_bytes, void *stream);

/* The same split for callers that cannot allocate device memory (no counterpart in the paper:
 * this is a packaging variant of pact_prune, not a step of the method).  pact_prune needs a
 * workspace that somebody obtained from cudaMalloc; a host that runs inside another framework's
 * callback, a plugin that is handed tensors but no allocator, or a process whose device memory is
 * already fully parcelled out cannot provide one.  This entry point takes no context and no
 * workspace, holds no device memory and calls no allocating routine; calls are independent of one
 * another (any streams, any threads) and may be captured.
 *  - N must not exceed PACT_PRUNE_STATIC_MAX_N, a limit of this interface (pact_prune has none); larger
 *    N returns PACT_ERR_UNSUPPORTED and launches nothing.  Only p->lambda and p->n_prune are read.
 * Inputs, outputs and their meaning are those of pact_prune. */
#define PACT_PRUNE_STATIC_MAX_N 65536
pact_status pact_prune_static(const float *score, int N, const pact_params *p /*host*/, uint8_t *keep,
                              int32_t *kept_idx, int32_t *pruned_idx, int32_t *counts, void *stream);

/* DBDPC, Algorithm 2 (Eq. 5-7) on the rows idx[0..q) of K[N, d_k]:
 * all-pairs cosine distance, density with d_n, density-ordered centre selection under d_c
 * (the result of the sequential loop, computed by asynchronous parallel resolution, cf.
 * Algorithm 4 / Appendix D), nearest-centre assignment.
 * idx must be ascending; q is read from q_dev (device int32).
 * Writes rho[q] (in idx order), center_idx[C] (token indices, ascending), C_dev,
 * label[N] (cluster id for rows in idx, -1 elsewhere), and counters (may be NULL). */
pact_status pact_dbdpc(pact_ctx *ctx, const void *K, int64_t ldK, int N, const int32_t *idx,
                       const int32_t *q_dev, const pact_params *p /*host*/, float *rho,
                       int32_t *center_idx, int32_t *C_dev, int32_t *label, int32_t *counters,
                       void *ws, size_t ws_bytes, void *stream);

/* Reincorporation, Eq. 8-9 / Algorithm 3 step 3: each row pruned_idx[0..m) of K joins its
 * nearest centre iff that distance is < alpha * d_c.  Updates label[N] in place for those rows
 * (cluster id or -1) and writes r_dev (number that joined).  counters may be NULL. */
pact_status pact_reincorporate(pact_ctx *ctx, const void *K, int64_t ldK, int N,
                               const int32_t *pruned_idx, const int32_t *m_dev,
                               const int32_t *center_idx, const int32_t *C_dev,
                               const pact_params *p /*host*/, int32_t *label, int32_t *r_dev,
                               int32_t *counters, void *ws, size_t ws_bytes, void *stream);

/* Choice of the reduction layer L (the paragraph that follows Eq. 11 and the figure it cites): the
 * earliest layer whose visual keys are spread widely enough.  K_layers is a HOST array of n_layers
 * DEVICE pointers, each a [N, n_kvh*d_h] key matrix with row stride ldK elements (keys before the
 * rotary embedding, as in that figure).  For every layer l, max_dist[l] (device, [n_layers]) receives
 * the largest cosine distance (Eq. 5) between two of its N keys, 0 when N = 1; layer_out (device,
 * [1], may be NULL) receives the smallest l with max_dist[l] >= threshold, or -1 when no layer
 * qualifies.  Distances are formed in the arithmetic of pact_dbdpc (fp32 for bf16 keys, fp64 rounded
 * to fp32 for fp32 keys).  ws must hold pact_workspace_bytes(ctx, min(n_layers, 16), N) bytes.
 * Asynchronous on `stream`; INVALID_ARG for null or misaligned pointers, n_layers < 1, N < 1, a bad
 * stride or a NaN threshold, before anything is launched. */
pact_status pact_key_spread(pact_ctx *ctx, const void *const *K_layers /*host*/, int n_layers, int64_t ldK,
                            int N, float threshold, float *max_dist, int32_t *layer_out, void *ws,
                            size_t ws_bytes, void *stream);

/* Merge, Eq. 10 / Algorithm 3 step 4: H_out row (vis_start + c) = mean of the visual rows of H
 * whose label is c (fp32 accumulation in ascending token order), P_out = position id of the
 * centre, size_out = members, logw_out = log(members) when given (the bias log W that Eq. 11
 * adds to the attention logits of the reduced sequence; 0 for text rows); text rows are copied
 * around the merged span.
 * Uses img->H, P, H_out, P_out, size_out, logw_out, counters (N_OUT and STATUS are written, the rest is zero).
 * label[i] must lie in [-1, C) and *C_dev in [0, N]; center_idx[c] in [0, N).  A label outside that
 * range is treated as -1 and reported as PACT_ERR_INVALID_ARG in counters[PACT_CNT_STATUS]; the other
 * rows are merged as usual. */
pact_status pact_merge(pact_ctx *ctx, const pact_image *img /*host*/, const int32_t *label,
                       const int32_t *center_idx, const int32_t *C_dev, const pact_params *p /*host*/,
                       void *ws, size_t ws_bytes, void *stream);

/* ---- the whole step over a batch (Algorithm 3) ------------------------------------------ */

/* imgs: host array of B images (independent units).  params: one pact_params for all
 * (params_stride = 0) or one per image (params_stride = 1).  All outputs named in pact_image
 * are written; nothing is read back to the host. */
pact_status pact_reduce(pact_ctx *ctx, const pact_image *imgs /*host*/, int B,
                        const pact_params *params /*host*/, int params_stride, void *ws,
                        size_t ws_bytes, void *stream);

/* ---- replayable form of pact_reduce (CUDA graph) --------------------------------------------- */

/* Records the launch sequence of pact_reduce(ctx, imgs, B, params, params_stride, ws, ws_bytes) once
 * into a CUDA graph; pact_graph_launch replays it on `stream` at a fraction of the launch cost (the
 * path is a chain of short dependent kernels, so launch gaps matter).  The graph holds the pointers
 * given here: the buffers and the workspace must stay valid and in place while it is used; their
 * contents may change between launches.  One launch at a time per graph (they share the workspace).
 * Nothing runs on the device during pact_graph_create. */
typedef struct pact_graph pact_graph;
pact_status pact_graph_create(pact_ctx *ctx, const pact_image *imgs /*host*/, int B,
                              const pact_params *params /*host*/, int params_stride, void *ws,
                              size_t ws_bytes, pact_graph **graph);
pact_status pact_graph_launch(pact_graph *graph, void *stream);
pact_status pact_graph_destroy(pact_graph *graph);

/* Same computation with HOST buffers for one image: copies the inputs to the device, runs
 * pact_reduce, brings H_out/P_out/size_out/logw_out/label/counters back (results in mapped host memory are
 * written there by the kernels) and synchronises.
 * From the second call of a context with hidden states of 12 MB or more on, they arrive while the queries are scored, on a
 * stream of the context's own: that call creates it (about 65 us, once) and pact_destroy gives it back.
 * dev_staging is a device buffer the caller provides (size from
 * pact_host_staging_bytes); every pointer inside `img` is a host pointer here. */
pact_status pact_reduce_host(pact_ctx *ctx, const pact_image *img /*host, host pointers*/,
                             const pact_params *p /*host*/, void *dev_staging, size_t staging_bytes,
                             void *ws, size_t ws_bytes, void *stream);
size_t pact_host_staging_bytes(const pact_ctx *ctx, int n_total, int N);

/* ---- after the reduction: a paged cache and the attention of one new token over it --------------
 *
 * The layers above the reduction keep the reduced sequence (counters[PACT_CNT_N_OUT] rows, a number that only the device
 * knows) in a cache, and their attention adds log W (logw_out) to the logits, Eq. 11.  The four calls below are that cache:
 * pact_cache_plan gives the new rows of a batch of requests pages and slots, pact_cache_write puts keys, values and biases into
 * them, pact_page_select finds the pages that a query may need most, and pact_paged_attention attends one new token per
 * request to all cached rows, or to those of the selected pages.  Lengths, counts and tables stay on the device, and every call may be
 * captured into a CUDA graph and replayed with other lengths in the same buffers.
 *
 * A page holds page_rows consecutive rows of one request (a multiple of 16, at most 1024).  Row p of request b lies in page
 * block_table[b][p / page_rows] at place p % page_rows; its slot is page * page_rows + place.
 *
 * `status` (device int32[1], may be NULL) is lowered to a negative pact_status when the device meets something that it cannot
 * serve, and never raised again: the caller clears it.  Whatever lengths, tables and slots hold, nothing outside the given buffers is read or
 * written.  The context's device must be the current one.  n_requests is at most PACT_MAX_REQUESTS.  Heads are at most 256 wide in bf16 and 128 in fp32
 * (PACT_ERR_UNSUPPORTED above). */
#define PACT_MAX_REQUESTS 4096

/* One layer's cache.  K and V: element [page][head][row][c] lies at page * k_page + head * k_head + row * k_row + c (elements;
 * multiples of 16 bytes), so both orders of the axes of a page are served; element type `in`.  The other arrays are contiguous. */
typedef struct {
  void *K, *V;
  int64_t k_page, k_head, k_row;
  int64_t v_page, v_head, v_row;
  float *logw;          /* [n_pages][page_rows] what the attention adds to the logits of a row: log W of Eq. 11, minus infinity for a
                           row that must not be seen; NULL: nothing is added                       */
  void *bounds;         /* [n_pages][n_kvh][2][d_h], element type `in`: smallest and largest value of each coordinate of the page's
                           keys (an element that is not a number gives way to one that is); NULL: not kept */
  float *w_max;         /* [n_pages] largest logw of the page, 0 in a cache without logw; given if and only if bounds is */
  int32_t n_pages, page_rows;
} pact_paged_cache;

/* Block tables and slots of the rows that come next.  length[b] rows of request b are cached, n_new[b * n_new_stride] rows
 * (0 or more) are to follow: a count array of its own, or the N_OUT counters of a batch that pact_reduce has just written
 * (stride PACT_N_COUNTERS).  A negative count ends the request: its pages go back and its length becomes 0.
 * free_pages is a stack of page ids, its top at free_pages[*n_free - 1].  Ended requests push their pages first, by ascending request and
 * ascending place; then the others take pages off the top in the same order.  Page ids are taken as they are (the calls that read or write rows check them).
 * The tables and the stack of a call name no page twice: one that two requests share (pact_paged_attention may read it for both) goes back once for each that ends, and is
 * handed out as often.  A caller that shares pages ends these requests itself.
 * New rows are packed (row_stride 0: row i of request b is row_start[b] + i, and n_rows is what the caller has room for), or each request has
 * row_stride of them (row b * row_stride + i; n_rows = n_requests * row_stride).
 * A call that cannot be served as a whole changes nothing: length_out and n_free_out repeat the old values, row_start is 0, every
 * slot -1, and status becomes PACT_ERR_NO_PAGES (more pages needed than free) or PACT_ERR_INVALID_ARG (a length that is negative or, with
 * the new rows, more than max_pages hold; more new rows than n_rows or row_stride; n_free outside 0 .. n_pages, or above n_pages once
 * ended requests have pushed their pages). */
typedef struct {
  int32_t page_rows, n_pages; /* of the cache (the same for all layers)                             */
  int32_t n_requests, max_pages;
  int32_t *block_table;       /* [n_requests][max_pages]; entries of new pages are written, the others left alone */
  const int32_t *length;      /* [n_requests]                                                       */
  const int32_t *n_new;       /* [n_requests] with stride n_new_stride >= 1                         */
  int64_t n_new_stride;
  int32_t *free_pages;        /* [n_pages]; changes above the old top only                          */
  const int32_t *n_free;      /* [1]                                                                */
  int32_t *length_out;        /* [n_requests]; may be length                                        */
  int32_t *n_free_out;        /* [1]; may be n_free                                                 */
  int32_t *row_start;         /* [n_requests + 1] prefix sums of the counts; may be NULL            */
  int64_t *slot;              /* [n_rows] slot of every new row, -1 behind the last; may be NULL    */
  int64_t n_rows;
  int32_t row_stride;
  int32_t reserved;
  int32_t *status;
} pact_plan;
pact_status pact_cache_plan(pact_ctx *ctx, const pact_plan *p /*host*/, void *stream);

/* Rows into their slots: row r of K and V (element [r][head][c] at r * ld_row + head * ld_head + c, type `in`) and logw[r] go to slot[r]; a
 * negative slot is skipped, one that no page of the cache has is skipped and sets status to INVALID_ARG.
 * Slots of a call differ.  Where the cache keeps bounds, the rows of a page are neighbours in the call, in ascending slots without a gap, as
 * pact_cache_plan lays them out: a page whose place 0 is written begins new bounds, those of other pages are widened. */
typedef struct {
  const void *K, *V;
  int64_t ld_row, ld_head;
  const float *logw;          /* [n_rows]; NULL: 0; not read where the cache has no logw           */
  const int64_t *slot;        /* [n_rows]                                                           */
  int64_t n_rows;
  int32_t *status;
} pact_new_rows;
pact_status pact_cache_write(pact_ctx *ctx, const pact_paged_cache *cache /*host*/, const pact_new_rows *r /*host*/, void *stream);

/* One new token per request: what pact_page_select and pact_paged_attention take. */
typedef struct {
  const void *Q;              /* element [b][j][c] at b * ldQ + j * ldQh + c, type `in`             */
  int64_t ldQ, ldQh;
  const int32_t *block_table; /* [n_requests][max_pages]                                            */
  const int32_t *length;      /* [n_requests] cached rows, the new token's own among them           */
  int32_t n_requests, max_pages;
  int32_t *selected;          /* [n_requests][n_kvh][n_select] places in the block table: written by pact_page_select, read by
                                 pact_paged_attention (NULL: all pages)                             */
  int32_t n_select;
  int32_t n_first, n_last;    /* pact_page_select: pages that are always selected                   */
  float scale;                /* of the logits; 1 / sqrt(d_h) as a rule                             */
  void *out;                  /* pact_paged_attention: element [b][j][c] at b * ldO + j * ldOh + c, type `out` (pointer and
                                 strides: multiples of four elements)                               */
  int64_t ldO, ldOh;
  float *lse;                 /* [n_requests][n_qh]; may be NULL                                    */
  int32_t *status;
  void *ws;                   /* workspace, 256-byte aligned                                        */
  size_t ws_bytes;
} pact_query;

/* Bytes of device workspace that pact_page_select and pact_paged_attention need for at most max_requests requests and max_pages entries per
 * block table.  It needs no initialisation and keeps nothing between calls. */
size_t pact_paged_workspace_bytes(const pact_ctx *ctx, int max_requests, int max_pages);

/* Pages that the new token should attend to.  For a page with bounds lo, hi and every query head j of a key head,
 * scale * sum_c (q_c hi_c where q_c > 0, q_c lo_c where q_c < 0) + w_max is at least every logit scale * q.k + logw of its rows that is a number (scale > 0); the page's
 * score is the largest of these over the heads (a sum that is not a number is left out), in the order of double precision.  Selected are the first
 * n_first and the last n_last pages of the request, then those with the largest scores, ties to the lower page, n_select in all.
 * selected: their places in ascending order, -1 behind the last.  n_first, n_last >= 0, n_first + n_last <= n_select; max_pages <= 65536.  Lengths
 * outside 0 .. max_pages * page_rows are clamped and page ids outside the cache score minus infinity; both set status to INVALID_ARG (ids only where
 * scores decide: a request with no more pages than n_select has all of them selected and none looked at). */
pact_status pact_page_select(pact_ctx *ctx, const pact_paged_cache *cache /*host*/, const pact_query *q /*host*/, void *stream);

/* Attention of the new token over its request's cached rows (Eq. 11): with s_p = scale * q.k_p + logw_p over the rows p in
 * 0 .. length[b] - 1, out = sum_p exp(s_p - lse) v_p and lse = log sum_p exp(s_p), for every query head, which reads key head
 * floor(j * n_kvh / n_qh).  With `selected` only the rows of those pages count: of the first min(n_select, pages of the request) entries,
 * those below 0 or beyond the request's pages are skipped, and a page named twice counts twice.  Rows with logw = minus infinity and
 * rows past the length have no effect, whatever their keys and values hold.  Without any row out is 0 and lse minus infinity.  Infinities and NaN in rows that count
 * leave infinities or NaN in the results that they enter (an infinite value beside bf16 keys: NaN).  Keys and values are read once for every 16 query heads of a key head (fp32: 8).
 * Logits, probabilities, softmax statistics and sums are fp32 (beside bf16 values probabilities are carried as three bf16 terms).
 * Lengths are clamped to 0 .. max_pages * page_rows and rows of pages outside
 * the cache are left out; both set status to INVALID_ARG. */
pact_status pact_paged_attention(pact_ctx *ctx, const pact_paged_cache *cache /*host*/, const pact_query *q /*host*/, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PACT_H_ */
