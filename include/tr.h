/*
 * tr.h -- C ABI of the ALTR visual-token reducer for GB300 (sm_103a).
 *
 * ALTR (arxiv 2607.13500, Section IV) keeps K of the N visual tokens of an
 * image: the K1 = floor(lambda K) tokens with the highest second-order Renyi
 * entropy of their channel-magnitude distribution (Stage I, Eq. 3-4), plus
 * K2 = K - K1 tokens taken at a fixed stride along the remaining tokens sorted
 * by the cosine between the final-layer MLP input x' and output x'' (Stage II,
 * Eq. 5-6), returned as X* = X_imp union X_div (Eq. 7, Algorithm 1).
 *
 * Conventions shared by every entry point:
 *  - Device pointers are owned by the caller; the library never allocates
 *    device memory, frees it or synchronises.  Every call enqueues work on
 *    `stream` (a cudaStream_t; NULL is the legacy default stream) and returns
 *    at once.  (A tr_pipeline owns host-side CUDA events, see below.)
 *  - The device of `stream` and of the pointers is the current one (a NULL
 *    stream names no device, and launch shapes follow the current device's
 *    SM count); the Python binding makes its tensors' device current itself.
 *  - Host-detectable errors (null or misaligned pointers, bad sizes, too small
 *    a workspace) are returned before anything is launched; outputs are left
 *    untouched.  A launch failure returns TR_ERR_CUDA.
 *  - Data-dependent conditions are counted in the optional device status
 *    words (int32[TR_STATUS_WORDS], accumulated with atomics; zero them before
 *    the call): [0] rows found to hold a non-finite value in an input the
 *    selection (or a requested H2 / s output) needed, [1] rows whose
 *    exact sums did not fit the exact representation (ordering of such a row
 *    falls back to its float key), [2] rows recomputed exactly to settle a
 *    near-tie, [3] images skipped because their budget was invalid
 *    (K < 0, K > N, K1 < 0 or K1 > K).
 *  - Kept indices are local to their image, ascending, and image b's
 *    occupy positions [cu_k[b], cu_k[b+1]) of `idx` and of `y`.
 *  - Ties go to the lower token index, in the top-K1 and in the sort.
 *  - The library keeps no global state besides two per-device caches (the
 *    "shared memory limit already raised" flags and the SM count, both
 *    atomic); calls from several host threads or on different streams may
 *    run concurrently when they use different workspaces and outputs.
 *  - The single-call entry points only enqueue kernels (no allocation,
 *    synchronisation or copies), so they can be captured into a CUDA graph
 *    and replayed; make one call on the device outside the capture first
 *    (it raises the kernels' shared-memory limit once).
 *  - tr_select, tr_gather, tr_select_gather and tr_reduce launch their
 *    kernels with programmatic dependent launch: a kernel may be scheduled
 *    while the kernel before it on the stream finishes, and waits in
 *    hardware for that kernel's completion before it reads anything, so
 *    stream order is kept (tr_score's kernel lets such a successor in as
 *    soon as all its CTAs run).  The pipeline launches normally.
 */
#ifndef TR_H
#define TR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TR_OK = 0,
  TR_ERR_ARG = 1,         /* null pointer, negative or inconsistent size       */
  TR_ERR_BUDGET = 2,      /* K > N, lambda or ratio outside [0, 1] (host)      */
  TR_ERR_DTYPE = 3,       /* dtype not one of tr_dtype                         */
  TR_ERR_ALIGN = 4,       /* d * sizeof(elem) % 16 != 0 or a base not 16-B aligned */
  TR_ERR_WORKSPACE = 5,   /* workspace NULL, too small or not 256-B aligned    */
  TR_ERR_CUDA = 6,        /* a kernel launch failed                            */
  TR_ERR_UNSUPPORTED = 7  /* N_b > TR_MAX_N or d > TR_MAX_D                    */
} tr_status;

typedef enum { TR_F32 = 0, TR_BF16 = 1, TR_F16 = 2 } tr_dtype;

#define TR_MAX_N 16384        /* tokens per image (keys of one image stay in shared memory) */
#define TR_MAX_D 16384        /* channels per token                                  */
#define TR_STATS_WORDS 8      /* fp32 words of the per-row statistics record         */
#define TR_STATUS_WORDS 4

/*
 * The token tensors of a batch of images, packed row-major as [total, d]:
 * image b owns rows [cu_seqlens[b], cu_seqlens[b+1]) (ragged), or
 * [b*n, (b+1)*n) when cu_seqlens is NULL (uniform).
 */
typedef struct {
  const void *x;              /* visual tokens X, the Stage-I input and gather source (Sec. III-A) */
  const void *x_pre;          /* final-layer MLP input x' (Eq. 5); NULL means x' = x               */
  const void *x_post;         /* final-layer MLP output x'' (Eq. 5); required                      */
  int32_t dtype;              /* tr_dtype of all three tensors                                     */
  int32_t d;                  /* channels D                                                         */
  int32_t batch;              /* images B                                                           */
  int32_t n;                  /* tokens per image N when cu_seqlens is NULL                         */
  const int32_t *cu_seqlens;  /* device int32[batch+1] row offsets, or NULL                         */
  int32_t total;              /* total rows T (ragged: must equal cu_seqlens[batch])                */
  int32_t max_n;              /* ragged: max_b N_b (host-known); ignored when uniform              */
  int32_t flags;              /* selection options, 0 or TR_STRIDE_INTERVAL                         */
} tr_tokens;

/*
 * Positions of the diversity picks along X_rem sorted by s (M = |X_rem|):
 *   flags = 0:                  Algorithm 1, the integer stride
 *                               t = max(1, floor(M / K2)): 0, t, ..., (K2-1) t;
 *   flags = TR_STRIDE_INTERVAL: the fixed interval (N - |X_imp|) / K2 = M / K2
 *                               of Section IV-B taken as a real number:
 *                               floor(j M / K2) for j < K2.
 * Both pick K2 distinct positions; they agree whenever K2 divides M.
 */
#define TR_STRIDE_INTERVAL 1

/* Name of a status code (static string). */
const char *tr_status_string(int32_t status);

/* Library version string. */
const char *tr_version(void);

/*
 * Budgets of Algorithm 1, first step, and Eq. 7 (host only, no device work).
 * Per image b with N_b = h_seqlens[b] tokens:
 *   K_b  = k                          when k > 0,
 *        = max(1, floor(N_b r_num / r_den)) (0 if N_b = 0) when k <= 0;
 *   K1_b = floor(K_b lam_num / lam_den), K2_b = K_b - K1_b;
 *   h_cu_k[0] = 0, h_cu_k[b+1] = h_cu_k[b] + K_b.
 * lambda = lam_num / lam_den must lie in [0, 1] (the paper's split of K = 192
 * into 64 + 128 tokens, Section V-C, is lambda = 1/3).  Returns TR_ERR_BUDGET
 * when K_b > N_b, a ratio lies outside (0, 1] or lambda outside [0, 1];
 * TR_ERR_ARG for null pointers or batch < 0.  h_k, h_k1: int32[batch];
 * h_cu_k: int32[batch+1].
 */
tr_status tr_budgets(int32_t batch, const int32_t *h_seqlens, int32_t k, int32_t r_num, int32_t r_den,
                     int32_t lam_num, int32_t lam_den, int32_t *h_k, int32_t *h_k1, int32_t *h_cu_k);

/* Device workspace bytes that tr_select and tr_reduce need for `in`
 * (0 on invalid input).  The workspace must be 256-byte aligned. */
size_t tr_workspace_bytes(const tr_tokens *in);

/*
 * Scoring pass (Eq. 3, 4 and 6 for every token): one read of x, x', x''.
 *   stats: device fp32[total, TR_STATS_WORDS] (16-byte aligned), per row
 *          [0] L1 = sum_j |x_j|, [1] S2 = sum_j x_j^2, [2] A = sum_j x'_j^2,
 *          [3] B = sum_j x''_j^2, [4] P_hi, [5] P_lo with P = sum_j x'_j x''_j
 *          = P_hi + P_lo (double-float), [6] the importance key L1^2 / S2
 *          and [7] the consistency key P / sqrt(A B), both rounded once to
 *          fp32 and NaN when the row's sums left the fp32 error model
 *          (non-finite, or S2, A or B outside [2^-100, 2^100]).  L1, S2, A, B
 *          are fp32 sums of bounded rounding depth; P is accumulated
 *          error-free up to a ~1e-10 relative residue.
 *   h2:    device fp32[total] or NULL: H2 = -log sum_j p_j^2 = log(L1^2 / S2)
 *          (Eq. 3-4); 0 for an all-zero row.
 *   s:     device fp32[total] or NULL: s = P / sqrt(A B) (Eq. 6); 0 when
 *          x' or x'' is all zero.
 * h2 and s come from the fp32 sums; rows whose sums overflow fp32 (inputs
 * above ~2^63 in magnitude) or hold non-finite inputs get non-finite values
 * here and are settled exactly by tr_select / tr_reduce.
 */
tr_status tr_score(const tr_tokens *in, float *stats, float *h2, float *s, void *stream);

/*
 * Selection (Stage I top-K1, Stage II sort and stride pick, Algorithm 1)
 * from the statistics of tr_score.  Decisions are exact: keys whose float
 * bounds overlap are recomputed from the inputs in exact integer arithmetic,
 * so the result is the selection defined by the real-valued H2 and s with
 * the lower-index tie-break.
 *   d_k, d_k1:  device int32[batch] budgets K_b, K1_b (see tr_budgets).
 *   d_cu_k:     device int32[batch+1] prefix sums of K_b.
 *   idx:        device int32[cu_k[batch]] kept local indices (ascending).
 *   role:       device uint8[total] or NULL: 0 dropped, 1 X_imp, 2 X_div.
 *   h2, s:      device fp32[total] or NULL: when given, rows whose fp32 sums
 *               were unreliable (non-finite, overflowed or underflowed) and
 *               rows recomputed for a near-tie get H2 / s rewritten from the
 *               exact sums (-inf H2 / +inf s for non-finite inputs).
 *   ws:         device workspace of tr_workspace_bytes(in) bytes.
 *   d_status:   device int32[TR_STATUS_WORDS] or NULL.
 */
tr_status tr_select(const tr_tokens *in, const float *stats, const int32_t *d_k, const int32_t *d_k1,
                    const int32_t *d_cu_k, int32_t *idx, uint8_t *role, float *h2, float *s, void *ws,
                    size_t ws_bytes, int32_t *d_status, void *stream);

/*
 * Gather of the kept tokens (Eq. 7: X* holds the original token vectors):
 * y[r] = x[first row of image b + idx[r]] for cu_k[b] <= r < cu_k[b+1], a
 * bit copy of d elements in the input dtype.
 *   d_cu_k:   device int32[batch+1] prefix sums of K_b (as for tr_select).
 *   idx:      device int32[total_k] local kept indices (tr_select's output).
 *   total_k:  host int, = cu_k[batch].
 *   y:        device [total_k, d] in the input dtype, 16-byte aligned.
 * A row whose index falls outside its image's tokens is written as zeros.
 */
tr_status tr_gather(const tr_tokens *in, const int32_t *d_cu_k, const int32_t *idx, int32_t total_k, void *y,
                    void *stream);

/*
 * Selection and gather in one launch, from the statistics of tr_score: the
 * result of tr_select (idx, optional H2 / s fix-ups, status) plus the kept
 * rows y as tr_gather would copy them.  When there are fewer images than
 * SMs, each image's selection is run by several CTAs at once and each copies
 * its share of the kept rows (the selection is deterministic, so all reach
 * the same indices; only one writes idx and the status words).
 *   total_k:  host int, = cu_k[batch]; y: device [total_k, d], 16-byte aligned.
 *   Other arguments as in tr_select (role is not produced).
 */
tr_status tr_select_gather(const tr_tokens *in, const float *stats, const int32_t *d_k, const int32_t *d_k1,
                           const int32_t *d_cu_k, int32_t total_k, void *y, int32_t *idx, float *h2, float *s,
                           void *ws, size_t ws_bytes, int32_t *d_status, void *stream);

/*
 * The whole path in one call on `stream`, with the statistics kept in the
 * workspace: tr_score then tr_select_gather for a uniform batch (two kernel
 * launches); tr_score, tr_select and tr_gather for a ragged one (three).
 *   total_k:  host int, = cu_k[batch] (the number of output rows).
 *   y:        device [total_k, d] in the input dtype, 16-byte aligned.
 *   idx, h2, s, d_status: as in tr_select (role is not produced); h2 and s
 *             may be NULL.
 */
tr_status tr_reduce(const tr_tokens *in, const int32_t *d_k, const int32_t *d_k1, const int32_t *d_cu_k,
                    int32_t total_k, void *y, int32_t *idx, float *h2, float *s, void *ws, size_t ws_bytes,
                    int32_t *d_status, void *stream);

/*
 * tr_reduce without a caller-provided workspace, for callers that cannot
 * allocate device memory (code running inside a host framework whose
 * allocator it cannot reach, plugins or callbacks that must not call
 * cudaMalloc, loops that must not allocate once they run).  The paper has
 * no counterpart: this is a deployment convenience of this library.
 *
 * Same arguments and results as tr_reduce, minus ws / ws_bytes.  Its scratch
 * is a device array of TR_NOALLOC_SCRATCH_BYTES bytes inside libtr, present
 * on every GPU that loads the library until the process exits; batches of
 * more than TR_NOALLOC_MAX_ROWS token rows are rejected with
 * TR_ERR_UNSUPPORTED.  The call allocates nothing.  The first call on a
 * device looks up that array's device address (with the device current),
 * so make the first call on each device before any stream capture.  All
 * calls share the array: calls whose work may overlap on the GPU race and
 * must be serialised by the caller.
 */
#define TR_NOALLOC_MAX_ROWS 32768
#define TR_NOALLOC_SCRATCH_BYTES (8u << 20)
tr_status tr_reduce_noalloc(const tr_tokens *in, const int32_t *d_k, const int32_t *d_k1, const int32_t *d_cu_k,
                            int32_t total_k, void *y, int32_t *idx, float *h2, float *s, int32_t *d_status,
                            void *stream);

/*
 * Overlapped reduction of successive batches, a stream pipeline over `slots`
 * slots.  Submission i uses slot i mod slots: it scores its batch on
 * score_streams[slot] (tr_score), then selects (tr_select) and gathers
 * (tr_gather) it on `select_stream`, which waits for that scoring only (a
 * uniform batch of one or two images of at most 1024 tokens is selected and
 * gathered by one tr_select_gather launch instead).  So
 * the selection and gather of one batch run while the next batch is scored,
 * and with a score stream per slot one batch's scoring starts while the
 * previous score kernel drains.  Give `select_stream` the higher priority:
 * the score kernel's CTAs retire one by one, and a higher-priority kernel
 * takes the SMs they free.  The slot's workspace ws[slot] (ws_bytes >=
 * tr_workspace_bytes bytes, 256-byte aligned, owned by the caller) is reused
 * only after the submission that used it last has been gathered (the score
 * stream waits for it).
 *
 * Ordering the caller keeps: the inputs of a submission (x, x', x'') stay
 * unchanged, and its outputs (y, idx, h2, s, d_status) untouched by other
 * work, until select_stream has passed the submission -- give each
 * submission still in flight its own output buffers (one set per slot).
 * Work that consumes a submission's outputs orders itself after it on
 * select_stream (or tr_pipeline_wait).
 *
 * The pipeline owns 3 x slots CUDA events, created on the current device by
 * tr_pipeline_create (make it the device of every stream) and destroyed by
 * tr_pipeline_destroy; it allocates no device memory and never synchronises.
 * One host thread at a time may submit to a pipeline (it keeps a count).
 *   tr_pipeline_create: score_streams holds `slots` cudaStream_t (they may
 *     repeat one stream); ws holds `slots` workspaces.
 *   tr_pipeline_submit: arguments as in tr_reduce, except that d_status is
 *     zeroed by the call itself (on select_stream, before the selection);
 *     score_begin / score_end are optional cudaEvent_t (or NULL) recorded on
 *     the slot's score stream right before and after the score kernel, to
 *     time it (as event-record nodes when the stream is being captured).
 *     Host-detectable errors are returned before anything is enqueued.
 *   tr_pipeline_wait: makes `stream` wait for every submission so far.
 *   tr_pipeline_kernels: kernels launched by the submissions so far (three
 *     per submission -- score, select, gather -- or two when a tiny uniform
 *     batch is selected and gathered in one launch); 0 for NULL.
 *
 * Graph capture: submissions made while the streams are captured into a
 * CUDA graph (forked from the capturing stream, joined back with
 * tr_pipeline_wait and a wait on each score stream) become one graph whose
 * replay runs those steps, overlapped as above, with a single launch.  Use a
 * pipeline created for the capture (no submission before it: the first
 * `slots` submissions of a pipeline wait on no earlier event) and only
 * replay it afterwards.
 */
#define TR_PIPELINE_MAX_SLOTS 8
typedef struct tr_pipeline tr_pipeline;
tr_status tr_pipeline_create(void *const *score_streams, void *select_stream, int32_t slots, void *const *ws,
                             size_t ws_bytes, tr_pipeline **out);
tr_status tr_pipeline_submit(tr_pipeline *p, const tr_tokens *in, const int32_t *d_k, const int32_t *d_k1,
                             const int32_t *d_cu_k, int32_t total_k, void *y, int32_t *idx, float *h2, float *s,
                             int32_t *d_status, void *score_begin, void *score_end);
tr_status tr_pipeline_wait(tr_pipeline *p, void *stream);
long long tr_pipeline_kernels(const tr_pipeline *p);
tr_status tr_pipeline_destroy(tr_pipeline *p);

/*
 * ---- The encoder's final-layer MLP with the scoring fused in (Eq. 5) ----
 *
 * Section IV-B takes x' (the input of the vision encoder's last MLP) and
 * x'' = f(x') = W2 sigma(W1 x') (its output, Eq. 5) from the encoder's
 * forward pass.  These two calls run that MLP on the tensor cores, and the
 * second one scores every token in its epilogue, so the selection needs no
 * separate pass over x, x', x'':
 *
 *   tr_mlp_hidden:  H = sigma(x' W1^T + b1)                       [t, d_hidden]
 *   tr_mlp_score:   x'' = H W2^T + b2, rounded to bf16 and stored  [t, d]
 *                   x   = resid + x'' (the block's output tokens X, the
 *                         Stage-I input and gather source), rounded to bf16
 *                         and stored; x = x'' when resid is NULL
 *                   stats: the per-row record of tr_score, with its sums
 *                         taken over the stored x, x' and x''.
 *
 * tr_select (or tr_select_gather) then takes tokens {x, x', x''} and these
 * stats exactly as it takes tr_score's; the result is the selection defined
 * by the stored tensors.  The sums of each record carry less rounding than
 * tr_score's (every term enters through TwoSum), within the same
 * certification bounds.
 *
 * Operands and outputs are bf16, row-major, 16-byte aligned; d and d_hidden
 * are multiples of 16.  Accumulation is fp32 in tensor memory; sigma is
 * evaluated in fp32 on the accumulator plus b1 and rounded once to bf16.
 * d_error (optional device int32, zero it first) gets a non-zero bit when a
 * pipeline wait inside the kernel timed out (not expected in a correct run;
 * the kernel then stops early and its outputs are incomplete).
 */
#define TR_ACT_GELU 0        /* x Phi(x), the erf form                        */
#define TR_ACT_QUICK_GELU 1  /* x / (1 + exp(-1.702 x)), CLIP's variant        */
#define TR_ACT_NONE 2
#define TR_MLP_MAX_HIDDEN 65536
typedef struct {
  const void *x_pre;   /* [t, d] bf16: the MLP input x' (Eq. 5)                        */
  const void *resid;   /* [t, d] bf16 added to x'' to form x, or NULL (x = x'')        */
  const void *w1;      /* [d_hidden, d] bf16 (nn.Linear layout)                        */
  const void *w2;      /* [d, d_hidden] bf16                                           */
  const float *b1;     /* [d_hidden] fp32 or NULL                                      */
  const float *b2;     /* [d] fp32 or NULL                                             */
  int32_t t;           /* rows (tokens of the whole batch)                              */
  int32_t d;           /* channels D                                                    */
  int32_t d_hidden;    /* hidden width of the MLP                                       */
  int32_t act;         /* sigma: TR_ACT_GELU, TR_ACT_QUICK_GELU or TR_ACT_NONE          */
} tr_mlp;

/* H = sigma(x' W1^T + b1): h is device bf16 [t, d_hidden]. */
tr_status tr_mlp_hidden(const tr_mlp *m, void *h, int32_t *d_error, void *stream);

/* Scratch bytes of tr_mlp_score (256-byte aligned device memory); 0 on invalid input. */
size_t tr_mlp_workspace_bytes(const tr_mlp *m);

/*
 * x'' = H W2^T + b2 and x = resid + x'' (both stored, bf16 [t, d]) with the
 * scoring of every row in the same pass: stats is device fp32
 * [t, TR_STATS_WORDS] laid out as in tr_score, h2 / s optional fp32 [t].
 * x_post and x must not overlap the inputs.
 */
tr_status tr_mlp_score(const tr_mlp *m, const void *h, void *x_post, void *x, float *stats, float *h2, float *s,
                       void *ws, size_t ws_bytes, int32_t *d_error, void *stream);

/*
 * ---- The first projector layer on the kept tokens, gathered on the fly ----
 *
 * The projector P maps the kept tokens X* = X_imp union X_div (Eq. 7) into
 * the LLM's embedding space (Z* = P(X*), Section III-A).  This call runs its
 * first layer, z = sigma(X* W^T + bias), on the tensor cores with the rows of
 * X* read straight from x by the selection's kept indices, so the gathered
 * copy y (tr_gather) is not needed for it:
 *   in:       the tokens x (bf16, as given to tr_select; x_pre / x_post unused)
 *   d_cu_k:   device int32[batch+1] prefix sums of K_b; idx: device int32
 *             [total_k] kept local indices (tr_select's output)
 *   w:        device bf16 [d_out, d] (nn.Linear layout); bias fp32 [d_out] or NULL
 *   act:      TR_ACT_GELU (LLaVA-1.5's projector), TR_ACT_QUICK_GELU, TR_ACT_NONE
 *   z:        device bf16 [total_k, d_out], row r for kept slot r
 * An index outside its image's tokens gives a row of zeros as input.  d and
 * d_out are multiples of 16; pointers 16-byte aligned.  d_error as for
 * tr_mlp_hidden.  Further projector layers are plain GEMMs on z.
 */
tr_status tr_project_kept(const tr_tokens *in, const int32_t *d_cu_k, const int32_t *idx, int32_t total_k,
                          const void *w, const float *bias, int32_t d_out, int32_t act, void *z, int32_t *d_error,
                          void *stream);

/*
 * The same first projector layer (Section III-A) on rows already gathered --
 * tr_gather's y, or any dense rows:
 *   y:        device bf16 [rows, d]
 *   w, bias, d_out, act: as for tr_project_kept
 *   z:        device bf16 [rows, d_out], row r from y's row r
 * z = sigma(y W^T + bias) by the kernel of tr_mlp_hidden; for y = the rows
 * that tr_project_kept reads, the two give the same z bit for bit (the same
 * MMA order and epilogue arithmetic).  Gathering first and projecting the
 * dense rows is the faster route on GB300: tr_project_kept's row loads are
 * TMA gathers whose issue rate sets its pace, while the copy costs one write
 * and one read of rows * d * 2 bytes.  d and d_out multiples of 16, pointers
 * 16-byte aligned; rows = 0 does nothing.  d_error as for tr_mlp_hidden.
 */
tr_status tr_project(const void *y, int32_t rows, int32_t d, const void *w, const float *bias, int32_t d_out,
                     int32_t act, void *z, int32_t *d_error, void *stream);

/*
 * ---- Into the language model: rotary positions and the paged cache ----
 *
 * The kept tokens Z* = P(X*) enter the LLM's attention layers (Section
 * III-A: E_l consumes Z* and the text).  These calls take one layer's
 * queries, keys and values from there to the attention output: the rotation
 * of queries and keys by positions with several axes (kept tokens are a
 * subset of their image's grid, so each token carries its own coordinates),
 * the append of keys and values to a paged cache, and the attention of the
 * new tokens over that cache.
 *
 * tr_heads: rows of one projection, element [t, h, c] at
 * p + t * token_stride + h * head_stride + c (strides in elements; the
 * channels are contiguous), so slices of a fused q/k/v projection pass as
 * they are.  Bases are 16-byte aligned, strides multiples of 16 bytes and
 * below 2^31 elements.
 */
typedef struct {
  void *p;               /* device; NULL where the argument is optional and absent */
  int64_t token_stride;  /* elements                                               */
  int64_t head_stride;
  int32_t heads;
} tr_heads;

/*
 * Rotary positions.  Frequency i < rot_dim / 2 turns one pair of channels by
 * the angle pos[axis[i]] * f_i: the pair (i, i + rot_dim / 2) with
 * TR_ROTARY_HALF, (2 i, 2 i + 1) with TR_ROTARY_PAIRS; channels >= rot_dim
 * keep their values.  turns[i] = f_i / (2 pi) * 2^64 modulo 2^64, an exact
 * fixed-point fraction of a turn: position times turns, modulo 2^64, is the
 * angle without any loss at large positions (int32, negative ones too).
 * tr_rotary_turns fills it on the host from the angular frequencies f_i.
 * head_dim and rot_dim are multiples of 8, rot_dim <= head_dim <= 256.  An
 * axis outside [0, axes) turns by nothing.
 */
#define TR_ROTARY_HALF 0
#define TR_ROTARY_PAIRS 1
#define TR_ROTARY_MAX_DIM 256
typedef struct {
  const uint64_t *turns;  /* device [rot_dim / 2] */
  const int32_t *axis;    /* device [rot_dim / 2] */
  int32_t head_dim, rot_dim;
  int32_t axes;           /* rows of pos          */
  int32_t layout;         /* TR_ROTARY_HALF or TR_ROTARY_PAIRS */
} tr_rotary;

/* Host only: h_turns[i] from h_freq[i] (radians per position, finite). */
tr_status tr_rotary_turns(const double *h_freq, int32_t n, uint64_t *h_turns);

/*
 * y = rotate(norm(x)) for every head of the queries and of the keys, in one
 * pass: norm(x) = x / sqrt(mean(x^2) + eps) * weight over the head's
 * channels where a weight (device fp32 [head_dim], 16-byte aligned, shared
 * by all heads) is given, x where it is NULL.  fp32 arithmetic, rounded once
 * into `dtype` (any tr_dtype), the type of all rows.
 *   pos:  device int32 [axes, tokens]
 *   q, q_out; k, k_out:  tr_heads of `tokens` rows; k and k_out may both be
 *         NULL.  Out may be the input itself (the same pointer and strides).
 */
tr_status tr_rotary_apply(const tr_rotary *r, int32_t dtype, int32_t tokens, const int32_t *pos, const tr_heads *q,
                          const float *q_weight, const tr_heads *q_out, const tr_heads *k, const float *k_weight,
                          const tr_heads *k_out, float eps, void *stream);

/*
 * The gradient of tr_rotary_apply: dq_out / dk_out with respect to q / k
 * from dq / dk with respect to its outputs, and where a weight is given its
 * gradient (device fp32 [head_dim], overwritten), the sum over all tokens
 * and heads taken in a fixed order (the same bits on every call on one GPU
 * model).  q and k (the forward inputs) are read only where their weight is
 * given and may be NULL otherwise.  ws: tr_rotary_backward_workspace_bytes
 * device bytes, 256-byte aligned (0 bytes, NULL allowed, without weights).
 */
size_t tr_rotary_backward_workspace_bytes(const tr_rotary *r, int32_t tokens);
tr_status tr_rotary_backward(const tr_rotary *r, int32_t dtype, int32_t tokens, const int32_t *pos,
                             const tr_heads *dq, const tr_heads *q, const float *q_weight, const tr_heads *dq_out,
                             float *dq_weight, const tr_heads *dk, const tr_heads *k, const float *k_weight,
                             const tr_heads *dk_out, float *dk_weight, float eps, void *ws, size_t ws_bytes,
                             void *stream);

/*
 * A paged key/value cache and one step's new tokens.  k and v are
 * [pages, heads, page, head_dim] in `dtype` (TR_BF16 or TR_F16); key j of
 * sequence b lies in page table[b, j / page] at slot j % page.  lens[b]
 * counts the keys of sequence b with the step's new tokens, which are its
 * last: new token t, cu_new[b] <= t < cu_new[b+1], is key
 * lens[b] - cu_new[b+1] + t.  All of this may change on the device between
 * replays of a captured graph; rows from cu_new[batch] on, if total_new is
 * larger, belong to no sequence (a graph captured for more tokens than a
 * replay has): they append nothing and attend to nothing.  page is a power
 * of two from 16 to 256, head_dim a multiple of 16 up to 128.  Nothing
 * outside the cache is touched whatever the device arrays hold: keys beyond
 * max_pages * page do not exist, a page id outside [0, pages) takes no append
 * and reads as zeros.  d_error (optional device int32, zero it first) then
 * gets TR_CACHE_ERR_PAGE (for the attention: if some row sees a key there;
 * pages before every window may be given away), or TR_CACHE_ERR_WAIT when a
 * pipeline wait inside the attention timed out (not expected in a correct
 * run; outputs incomplete).
 */
#define TR_CACHE_ERR_PAGE 1
#define TR_CACHE_ERR_WAIT 2
typedef struct {
  void *k, *v;             /* device [pages, heads, page, head_dim], 16-byte aligned */
  int32_t dtype;
  int32_t pages, heads, page, head_dim;
  const int32_t *table;    /* device [batch, max_pages] page ids   */
  int32_t batch, max_pages;
  const int32_t *lens;     /* device [batch]                       */
  const int32_t *cu_new;   /* device [batch + 1], cu_new[0] = 0    */
  int32_t total_new;       /* host: rows; cu_new[batch] at most    */
} tr_cache;

/*
 * Appends the new tokens' keys and values: k is normed (k_weight) and
 * rotated (r, pos) as in tr_rotary_apply on the way (r and k_weight may be
 * NULL), v is copied.  q, if given, holds the queries of the same tokens:
 * q_out = rotate(norm(q)) in the same launch.  All rows in the cache's dtype.
 */
tr_status tr_cache_append(const tr_cache *c, const tr_heads *k, const tr_heads *v, const tr_rotary *r,
                          const int32_t *pos, const float *k_weight, const tr_heads *q, const float *q_weight,
                          const tr_heads *q_out, float eps, int32_t *d_error, void *stream);

/*
 * Attention of the new tokens over the cache (their own keys appended
 * first): o[t, h] = sum_j p_j v_j with p = softmax(scale q[t, h] . k_j) over
 * the visible keys j of key head h / (q heads / key heads).  With
 * i = lens[b] - cu_new[b+1] + t the token's own key, key j is visible when
 *   0 <= j < lens[b],  j <= i if causal,  j > i - window if window > 0.
 * A row that sees no key (or only scores of -inf, or of no sequence) gives
 * zeros (lse = -inf).  A key that a row does not see takes no part in it,
 * whatever it holds.  (Values that are not finite cost a step little, however
 * long its sequences; only where max_len promises 512 keys at most are the
 * rows that one would spoil computed again, one by one, in 0.1 us a key.)
 * An infinite value that a row does see gives infinity in its channel, or NaN
 * where its probability rounds to zero.
 * Probabilities are rounded to the cache's type for their product with V;
 * their sum and everything else is fp32.
 *   q, o:     tr_heads of total_new rows, the same number of heads, a
 *             multiple of the cache's; o does not overlap q
 *   lse:      device fp32 [total_new, q heads] or NULL: log sum exp of the
 *             scaled scores
 *   max_new, max_len: what the host knows of a sequence's new tokens and of
 *             lens at most.  They only choose the launch (rows of a block,
 *             parts of the keys): a bound that is off costs time, no more
 *   ws:       device workspace of tr_cache_attend_workspace_bytes bytes,
 *             256-byte aligned
 */
size_t tr_cache_attend_workspace_bytes(const tr_cache *c, int32_t q_heads, int32_t window, int32_t max_new,
                                       int32_t max_len);
tr_status tr_cache_attend(const tr_cache *c, const tr_heads *q, const tr_heads *o, float *lse, float scale,
                          int32_t causal, int32_t window, int32_t max_new, int32_t max_len, void *ws,
                          size_t ws_bytes, int32_t *d_error, void *stream);

/*
 * ---- The paged cache held in 8 bits ----
 *
 * The same cache in half the bytes: c.k and c.v hold e4m3 codes (one byte,
 * [pages, heads, page, head_dim]), and every 16 keys of a head (a block)
 * share one scale 2^(e - 127), a byte e in k_scale / v_scale [pages, heads,
 * page / 16]: key j's channel c stands for code * scale.  c.dtype is the type
 * of the rows (queries, new keys and values, outputs: TR_BF16 or TR_F16);
 * everything else is as in tr_cache.
 *
 * tr_cache8_append: a block's scale is the least one that holds the finite
 * magnitudes of the rows it gets by the call (magnitude <= 448 * scale, 10 <=
 * e <= 246), and not below the block's old one if it has keys before the
 * call's; those keys are then coded anew by the scales' quotient, a power of
 * two, which rounds nothing but what falls under the codes' smallest step.
 * Codes are the nearest (ties to even, 448 at most); a value that is not
 * finite is held as NaN.  k_weight, r, pos, q as in tr_cache_append: norm and
 * rotation in fp32, rounded once into the codes.  Two sequences of a call may
 * not share a page that it writes.
 *   Tokens that are taken back later (drafts that are refused) leave the block
 * that they shared with older keys as they made it: with the larger scale, if
 * they needed one, and the older codes rounded for it.
 */
#define TR_CACHE8_BLOCK 16
typedef struct {
  tr_cache c;
  uint8_t *k_scale, *v_scale; /* device [pages, heads, page / 16] */
} tr_cache8;
tr_status tr_cache8_append(const tr_cache8 *c, const tr_heads *k, const tr_heads *v, const tr_rotary *r,
                           const int32_t *pos, const float *k_weight, const tr_heads *q, const float *q_weight,
                           const tr_heads *q_out, float eps, int32_t *d_error, void *stream);

/*
 * Attention over it: tr_cache_attend, with the keys and values that the codes
 * stand for.  Every e from 0 to 254 is taken as it stands (255 as 254).  The
 * products take codes, which fit exactly, queries and probabilities as halves:
 * bf16 queries in units of a power of two of each row's own, probabilities with
 * the values' scales on them: whole down to 2^-20, and lost below 2^-31, of the
 * greatest that the row sees (where blocks of zeros, held with e <= 10, count
 * with 2^-80 of the largest scale among the sequence's keys, if that is more than
 * theirs).  Sums are fp32.  So are the scores: a row with one
 * of 2^23 or more (or its negative), where fp32 no longer tells apart what
 * differs by one, gets no result to rely on.
 */
size_t tr_cache8_attend_workspace_bytes(const tr_cache8 *c, int32_t q_heads, int32_t window, int32_t max_new,
                                        int32_t max_len);
tr_status tr_cache8_attend(const tr_cache8 *c, const tr_heads *q, const tr_heads *o, float *lse, float scale,
                           int32_t causal, int32_t window, int32_t max_new, int32_t max_len, void *ws,
                           size_t ws_bytes, int32_t *d_error, void *stream);

/*
 * ---- Block tables kept on the device ----
 *
 * What a step of the paged caches goes by -- table, lens, cu_new -- built from
 * the tokens that each sequence gets, without the host: a stack of free pages
 * (free[0 .. *free_count), the next one to be taken last) and two calls.
 *
 * tr_pages_extend: sequence b gets d_new[b] tokens (negative: none).  cu_new
 * [batch + 1] becomes their prefix sums; the pages that the sequences grow
 * into are taken from the stack, sequence by sequence, and entered into the
 * table; lens grows; and each of the total_new rows gets the slot of its key
 * in the cache (page id * page + place in the page), its position in its
 * sequence and the sequence's number.  Rows behind the last token get -1 in
 * all three.
 *   A step that cannot be taken changes neither table, lens nor stack: cu_new
 * is zeros, all rows belong to no sequence, and d_error (optional device
 * int32, zero it first) gets TR_PAGES_ERR_FULL (not enough free pages),
 * TR_PAGES_ERR_LONG (a sequence would outgrow its row of the table),
 * TR_PAGES_ERR_ROWS (more tokens than total_new) or TR_PAGES_ERR_STATE (lens
 * or free_count are out of range).
 *
 * tr_pages_truncate: sequence b keeps its first d_keep[b] tokens at most
 * (negative: none); pages that hold none of these go back to the stack in the
 * opposite of the order in which they were taken, and their entries become -1.
 * Directly after an extend, to the lengths before it, table, lens and stack are
 * as they were (what was appended in between stays in the cache: see
 * tr_cache8_append for the block that it shares with older keys).  Refused as
 * above (TR_PAGES_ERR_STATE).
 *
 * Calls on one table come one after another (a stream, or events between
 * streams); all of it may be captured and replayed.  ticket is one int32 of
 * the calls' own, zero before the first.
 */
#define TR_PAGES_ERR_FULL 1
#define TR_PAGES_ERR_LONG 2
#define TR_PAGES_ERR_ROWS 4
#define TR_PAGES_ERR_STATE 8
typedef struct {
  int32_t *table;       /* device [batch, max_pages]  */
  int32_t *lens;        /* device [batch]             */
  int32_t *free;        /* device [pages]             */
  int32_t *free_count;  /* device [1]                 */
  int32_t *ticket;      /* device [1]                 */
  int32_t batch, max_pages;
  int32_t pages, page;  /* of the cache               */
} tr_pages;
tr_status tr_pages_extend(const tr_pages *p, const int32_t *d_new, int32_t total_new, int32_t *cu_new, int32_t *slots,
                          int32_t *pos, int32_t *seq, int32_t *d_error, void *stream);
tr_status tr_pages_truncate(const tr_pages *p, const int32_t *d_keep, int32_t *d_error, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* TR_H */
