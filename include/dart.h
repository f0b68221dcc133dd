/*
 * dart.h -- C ABI of the duplication-aware token reduction step (DART,
 * arXiv 2502.11494, Section 3.3) for AMD MI355X (gfx950).
 *
 * The step runs between two decoder layers of a multimodal LLM.  Per sample it
 *   (a) picks P pivot tokens by the largest L1 norm of a criterion row
 *       (Definition 1; Table 1 caption; the footnote of Section 3.3 that
 *       defines the K-norm as an L1 norm),
 *   (b) scores every token against every pivot with the cosine similarity of
 *       Definition 2 / Eq. (7),
 *   (c) retains the pivots plus, pivot by pivot, the tokens that duplicate that
 *       pivot least, until the keep budget is met (Eq. (9)-(10) with the
 *       per-pivot threshold fixed by the reduction ratio),
 *   (d) compacts hidden-state rows and position ids to the retained tokens in
 *       their original order, so the remaining layers run on the shorter
 *       sequence (Appendix D, post-pruning sequence length).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Memory.  `desc` is host memory, read during the call only; the device arrays it
 *   names (cu_seqlens, ext_pivots, span_start) are read by the enqueued kernels and must
 *   stay valid and unchanged until that work has finished.  Every other
 *   pointer is DEVICE memory owned by the caller unless stated otherwise.  The
 *   library never allocates, frees or keeps a pointer; scratch comes from the
 *   caller's workspace `ws` of at least dart_workspace_bytes(desc) bytes,
 *   256-byte aligned.  Inputs are never written.  Outputs must not alias inputs.
 * Layout.  X holds `total_N` token rows of D elements, row stride `ld`
 *   elements, sample after sample.  Dense: sample b owns rows [b*N, (b+1)*N).
 *   Ragged: sample b owns rows [cu_seqlens[b], cu_seqlens[b+1]).  Row starts
 *   must be 16-byte aligned (X base, ld*elemsize and D*elemsize multiples of 16).
 * Budget.  Sample b keeps K_b tokens: K_b = K if K > 0, otherwise
 *   K_b = floor(N_b * keep_num / keep_den).  P <= K_b <= N_b is required.
 *   keep/pos_out/Y are packed: sample b owns rows [cu_keep[b], cu_keep[b+1]),
 *   cu_keep[b] = sum of K_b' over b' < b (dense with K > 0: b*K).
 * Streams.  `stream` is a hipStream_t passed as void* (NULL = default stream).
 *   Calls only enqueue work; outputs are valid once the stream reaches that
 *   point.  No call synchronises except dart_device_status.
 * Errors.  Violations visible on the host return a negative dart_status and
 *   enqueue nothing.  In ragged mode the per-sample sizes live on the device:
 *   a sample with N_b > max_N, N_b < P, K_b < P or K_b > N_b (N_b == 0 is a
 *   valid empty sample), or whose span (desc.span_start) leaves X, is skipped -- it
 *   keeps zero tokens -- and a flag is raised in the workspace that
 *   dart_device_status reports.
 *   Non-finite input values give unspecified (but memory-safe) results.
 * Value range.  The fp32 arithmetic of the bf16 path (exact products of two bf16 values,
 *   32-term sums of them, row sums of |x| and x^2) must neither overflow nor lose bits to
 *   underflow, or the rounding bound the decisions are certified against does not hold:
 *   every non-zero element must satisfy 2^-55 <= |x| <= 2^55 (zeros are fine), for either
 *   dtype.  Inside that range a common power-of-two factor on a sample changes no output
 *   bit.  Outside it the retained set may differ from the exact one (memory-safe, not
 *   detected: the library does not scan its input).
 * Determinism.  Same inputs give bit-identical outputs, call after call, and a
 *   row's score depends only on its bytes and the pivot's bytes, not on where
 *   the row sits in the batch.  (Different entry points or pivot modes may take the
 *   token norms from different passes: their scores agree within
 *   dart_score_tolerance, not necessarily in the last bit.)
 * Limits.  B <= 2^20, 1 <= P <= 64, N_b <= 16384, D <= 65536, total_N <= 2^27, row strides (ld, crit_ld,
 *   ext_ld) <= 2^24 elements.
 * Pivots from outside (desc.P_ext > 0).  Tokens are scored against such a pivot and it
 *   has its stage in step (c) like any pivot -- after the pivots that are tokens, in the
 *   order of its rows -- but it is no token: it is never retained and holds no slot of
 *   the budget.  With P_in = P - P_ext, R starts as the P_in pivots inside the sample, the
 *   P stages share K_b - P_in slots (floor((K_b - P_in)/P) each, +1 for the first
 *   (K_b - P_in) mod P stages) and P_in <= K_b <= N_b is required instead of
 *   P <= K_b <= N_b.  In every piv array entry i >= P_in of a sample is not read; where
 *   the library writes piv it sets that entry to -1 - (i - P_in).  Step (a) chooses P_in
 *   pivots (none if P_ext == P).
 */
#ifndef DART_H_
#define DART_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define DART_API __attribute__((visibility("default")))
#else
#define DART_API
#endif

typedef enum dart_status {
  DART_OK = 0,
  DART_ERR_NULL = -1,      /* a required pointer is NULL                          */
  DART_ERR_SHAPE = -2,     /* B, N, D, P, ld, total_N or max_N out of range        */
  DART_ERR_BUDGET = -3,    /* P <= K <= N violated, or bad keep_num/keep_den       */
  DART_ERR_DTYPE = -4,     /* unknown dtype or pivot mode                          */
  DART_ERR_WORKSPACE = -5, /* ws NULL, misaligned or smaller than required         */
  DART_ERR_ALIGN = -6,     /* a row start would not be 16-byte aligned             */
  DART_ERR_HIP = -7,       /* a HIP call or kernel launch failed                   */
  DART_ERR_DEVICE = -8,    /* dart_device_status: a ragged sample or a given pivot
                              list was rejected on the device                      */
  DART_ERR_STATIC_LIMIT = -9 /* dart_reduce_static: the problem needs more scratch than
                              the library's built-in buffer holds                  */
} dart_status;

typedef enum dart_dtype {
  DART_F32 = 0,  /* IEEE binary32 hidden states                                    */
  DART_BF16 = 1  /* bfloat16 hidden states (upper half of a binary32)              */
} dart_dtype;

typedef enum dart_pivot_mode {
  DART_PIVOT_MAX_L1 = 0, /* largest criterion L1 norm first (Table 1 caption)      */
  DART_PIVOT_MIN_L1 = 1, /* smallest first (the "heart" rows of the pivot ablation) */
  DART_PIVOT_GIVEN = 2,  /* dart_reduce only: the caller supplies the pivots; see dart_reduce */
  DART_PIVOT_RANDOM = 3  /* dart_select_pivots and dart_reduce: drawn at random from desc.seed
                            (the random rows of the pivot ablation, Section 4.3 / Table 8).
                            The paper names no generator; the draw is defined here: sample
                            b draws tokens d_t = floor(w_t * N_b / 2^32), t = 0, 1, ..., where
                            w_t is word t mod 4 of the Philox4x32-10 block (Salmon et al.,
                            SC'11) with counter (t div 4, b, 0, 0) and key (low, high 32 bits
                            of seed); the sample's P - P_ext pivots are its first distinct
                            draws, in the order they appear, which is also their stage order
                            in step (c).  (After 4096 draws, which 64 pivots among 64 tokens
                            reach with probability below 1e-25, the lowest unused tokens
                            complete the list; DART_RANDOM_DRAW_LIMIT=n in the environment,
                            0 <= n <= 4096, lowers that limit so that a test can reach the
                            completion.)  No criterion is read: crit is ignored.            */
} dart_pivot_mode;

typedef enum dart_score_mode {
  DART_SCORE_PER_PIVOT = 0, /* Eq. (9)-(10) with a threshold per pivot: the staged rule  */
  DART_SCORE_MIN = 1,       /* one threshold for all pivots on min_i S[i][j]             */
  DART_SCORE_MAX = 2        /* one threshold for all pivots on max_i S[i][j]             */
} dart_score_mode;

/* Problem descriptor (host memory, plain data). */
typedef struct dart_desc {
  int32_t B;        /* samples in the batch, >= 0 (0 is a valid no-op)              */
  int32_t D;        /* hidden size: elements per token row                          */
  int32_t P;        /* pivots per sample (Definition 1), 1..64                      */
  int32_t N;        /* tokens per sample, dense layout; ignored when ragged         */
  const int32_t* cu_seqlens; /* DEVICE int32[B+1] row offsets, or NULL for dense    */
  int32_t total_N;  /* rows of X; dense: B*N (0 means "derive"); ragged: required   */
  int32_t max_N;    /* ragged: host-known upper bound of every N_b; dense: ignored  */
  int64_t ld;       /* row stride of X in elements, >= D                            */
  int32_t dtype;    /* dart_dtype of X, crit and Y                                  */
  int32_t K;        /* keep budget per sample (pivots included); 0 = use the ratio  */
  int32_t keep_num; /* K == 0: K_b = floor(N_b * keep_num / keep_den)               */
  int32_t keep_den;
  int32_t pivot_mode; /* dart_pivot_mode                                            */
  int32_t score_mode; /* dart_score_mode (0 = the default staged rule)              */
  /* Pivots from outside the scored tokens (the text-token pivots of the pivot ablation,
   * Table 8, and of the study of the pivots' modality): of the P pivots of every sample
   * the LAST P_ext are rows of ext_pivots, the first P - P_ext are tokens of the sample.
   * 0 = all pivots are tokens of the sample (then the two fields below are ignored).    */
  int32_t P_ext;
  int64_t ext_ld;         /* row stride of ext_pivots in elements, >= D                  */
  const void* ext_pivots; /* DEVICE rows [B*P_ext, D] of X's dtype, 16-byte aligned row
                             starts: sample b's outside pivot e is row b*P_ext + e        */
  /* Samples that are spans of a larger tensor (the vision tokens inside whole sequences of
   * text and vision tokens): with span_start != NULL (ragged layout required) sample b's
   * N_b = cu_seqlens[b+1] - cu_seqlens[b] tokens are rows span_start[b] .. span_start[b] +
   * N_b - 1 of X -- and of crit and pos, which are indexed like X -- and X has X_rows rows.
   * S, l1_out and keep stay packed by cu_seqlens.  A span that leaves [0, X_rows) makes its
   * sample a skipped one (see Errors).  NULL: the samples are packed back to back.        */
  const int32_t* span_start; /* DEVICE int32[B], or NULL                                   */
  int32_t X_rows;            /* rows of X when span_start != NULL (>= total_N)             */
  uint64_t seed;             /* DART_PIVOT_RANDOM: the seed of the draw (ignored otherwise) */
} dart_desc;

/* Bytes of workspace every entry point below accepts for this descriptor
 * (host arithmetic only; 0 if the descriptor is invalid). */
DART_API size_t dart_workspace_bytes(const dart_desc* desc);

/* The tile of the score kernel (step (b), Eq. 7) this library would use for the descriptor on
 * the current GPU (256 compute units assumed when there is none): *waves wavefronts per
 * workgroup in *split groups that share 16 * waves / split token rows and split the hidden
 * dimension among them; both 0 for fp32 descriptors, whose score kernel has one shape.  This
 * is the shape of dart_reduce with the hidden states as their own criterion.  Host
 * arithmetic only; waves and split are HOST pointers.  The choice is a cost model over the
 * batch's shape (see the library's source); DART_SCORE_TILE="W,KS" in the environment names
 * one of the built shapes instead, and a value that names none, or one whose tiles do not fit
 * the LDS with this many pivots, makes every entry point return DART_ERR_SHAPE.  The results of
 * the step do not depend on the shape (decisions are certified in fp64). */
DART_API dart_status dart_score_tile_shape(const dart_desc* desc, int32_t* waves, int32_t* split);

/* The same for calls whose score pass is the first pass over X: dart_reduce with a separate
 * criterion tensor (its norm pass reads crit, not X) and dart_duplication_scores.  Such calls
 * find no row of X in the memory-side cache, and small dense batches then do better with
 * four groups of waves per tile (measured; see the library's source).  For descriptors whose
 * pivots are given, drawn at random or all from outside, dart_score_tile_shape already
 * reports this shape (no norm pass over X exists for them). */
DART_API dart_status dart_score_tile_shape_first_read(const dart_desc* desc, int32_t* waves,
                                                      int32_t* split);

/* (a) Pivot selection -- Definition 1 with the max-L1-norm criterion of the
 * Table 1 caption.  crit: criterion rows [total_N, crit_D] with row stride
 * crit_ld (same dtype as X, e.g. the layer's key states), or NULL to use the
 * hidden-state rows themselves (then crit_D/crit_ld are ignored).
 * DART_PIVOT_RANDOM: the pivots are drawn from desc.seed instead (see dart_pivot_mode), in
 * draw order; crit is ignored and l1_out is not written.
 * Output piv[b*P + i] = index, local to sample b, of its i-th pivot, ordered by
 * (L1 norm descending, index ascending) -- ascending norm for DART_PIVOT_MIN_L1.
 * Norms are summed in fp64, in an order that depends on the row's length alone,
 * and ranked by these sums; rows of equal bytes tie.  l1_out (optional,
 * float[total_N]) receives the L1 norm of every criterion row, rounded once to fp32. */
DART_API dart_status dart_select_pivots(const dart_desc* desc, const void* X, const void* crit,
                               int32_t crit_D, int64_t crit_ld, int32_t* piv, float* l1_out,
                               void* ws, size_t ws_bytes, void* stream);

/* (b) Duplication scores -- Eq. (7): S = <p_i, x_j> / (|p_i| |x_j|), Euclidean
 * norms, 0 when either norm is 0.  piv as produced by dart_select_pivots.
 * S is pivot-major per sample: sample b, pivot i, token j at
 * S[P*row0(b) + i*N_b + j] with row0(b) the sample's first row in X.
 * bf16 inputs: exact bf16 products summed 32 at a time on the matrix cores in
 * fp32, those partial sums added in fp64; fp32 inputs: fp64 throughout.  The
 * stored value is rounded to fp32. */
DART_API dart_status dart_duplication_scores(const dart_desc* desc, const void* X, const int32_t* piv,
                                    float* S, void* ws, size_t ws_bytes, void* stream);

/* (c) Retained set -- Eq. (9)-(10).  R starts as the pivots; with m = K_b - P,
 * pivot i (in pivot order) adds the floor(m/P) (+1 for the first m mod P
 * pivots) not-yet-retained tokens of lowest S[i][.], ties to the lowest index.
 * keep receives each sample's retained indices (local to the sample) in
 * ascending order; cu_keep (optional, int32[B+1]) receives the packed offsets.
 * X == NULL: S is taken as exact.  X != NULL: wherever two fp32 scores at a
 * decision boundary are closer than the rounding bound of
 * dart_duplication_scores, the candidates involved are re-scored in fp64 from
 * the rows of X before deciding.
 * DART_SCORE_MIN / DART_SCORE_MAX: a second reading of Eq. (9)-(10), one threshold
 * common to all pivots: R = the pivots plus the K_b - P other tokens whose aggregate
 * score over the pivots (minimum or maximum) is lowest, ties to the lowest index. */
DART_API dart_status dart_topk_keep(const dart_desc* desc, const float* S, const int32_t* piv,
                           const void* X, int32_t* keep, int32_t* cu_keep, void* ws,
                           size_t ws_bytes, void* stream);

/* (d) Compaction -- the shortened sequence of Appendix D.  For sample b and
 * r < K_b: Y[cu_keep[b]+r][:] = X[row0(b)+keep[cu_keep[b]+r]][:] (D elements,
 * bit copy, Y rows densely packed with stride D) and
 * pos_out[cu_keep[b]+r] = pos[row0(b)+keep[...]].  pos/pos_out may both be NULL. */
DART_API dart_status dart_gather_compact(const dart_desc* desc, const void* X, const int64_t* pos,
                                const int32_t* keep, void* Y, int64_t* pos_out, void* ws,
                                size_t ws_bytes, void* stream);

/* (a)-(d) in one call.  Optional outputs (NULL to skip): pos/pos_out, cu_keep,
 * piv_out [B*P], S_out [P*total_N].  Y == NULL skips step (d) (pos/pos_out are then
 * ignored): for callers that compact whole sequences with dart_compact_sequences.
 * DART_PIVOT_GIVEN: step (a) is skipped and piv_out (required) is READ: piv_out[b*P + i]
 * is the index, local to sample b, of the pivot of stage i; crit is ignored.  The P
 * indices of a sample must be distinct and inside the sample: a list that is not makes
 * dart_device_status report DART_ERR_DEVICE and leaves that call's outputs unspecified
 * (nothing is read or written out of bounds).
 * DART_PIVOT_RANDOM: step (a) draws the pivots from desc.seed (see dart_pivot_mode) instead
 * of ranking norms; piv_out, if given, receives them; crit is ignored. */
DART_API dart_status dart_reduce(const dart_desc* desc, const void* X, const void* crit, int32_t crit_D,
                        int64_t crit_ld, const int64_t* pos, void* Y, int64_t* pos_out,
                        int32_t* keep, int32_t* cu_keep, int32_t* piv_out, float* S_out,
                        void* ws, size_t ws_bytes, void* stream);

/* dart_reduce for callers that already hold the criterion norms, e.g. from an epilogue of the
 * projection that produced the criterion rows (the K-norm of the Section 3.3 footnote computed
 * where the keys are computed): l1[j] (DEVICE float[total_N], packed like S) approximates the
 * L1 norm of criterion row j with a relative error of at most l1_rel_err (0 <= l1_rel_err <=
 * 0.1; the caller's promise, not checked; the rounding of an exact norm to fp32 is allowed for
 * on top of it).  The norm pass is skipped, so the hidden states
 * are read once, by the score pass.  The pivots are still those of the exact norms: every
 * token whose approximate norm could reach the top P within that error is re-evaluated in
 * fp64 from its criterion row (crit, or X when crit is NULL) and ranked by (exact norm, index),
 * so a loose bound costs time (more rows to re-read), a wrong one can cost the right pivots.
 * DART_PIVOT_MAX_L1 / DART_PIVOT_MIN_L1 only (DART_ERR_DTYPE otherwise); everything else as
 * dart_reduce. */
DART_API dart_status dart_reduce_with_norms(const dart_desc* desc, const void* X, const void* crit,
                                            int32_t crit_D, int64_t crit_ld, const float* l1,
                                            double l1_rel_err, const int64_t* pos, void* Y,
                                            int64_t* pos_out, int32_t* keep, int32_t* cu_keep,
                                            int32_t* piv_out, float* S_out, void* ws,
                                            size_t ws_bytes, void* stream);

/* dart_reduce for callers that cannot allocate device memory or hand over a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, results and kernels as dart_reduce, but the scratch memory is a buffer built
 * into the library (a file-scope device array of dart_static_scratch_bytes() bytes -- 32 MiB
 * -- that every GPU the library runs on holds until the process ends) instead of `ws`.  The
 * call allocates and frees nothing.
 *   - A descriptor whose dart_workspace_bytes() exceeds dart_static_scratch_bytes() is
 *     refused with DART_ERR_STATIC_LIMIT and nothing is enqueued (the five benchmark shapes
 *     except the 1.7 GB ragged batch fit).
 *   - All calls on one GPU share that GPU's buffer: two calls whose work overlaps in time on
 *     the same GPU (different streams, or threads) race on it.  Calls on one stream are safe.
 *   - dart_device_status for such a call: pass ws = NULL to dart_device_status_static.
 * The buffer keeps the previous call's contents; the kernels initialise every word they
 * read. */
DART_API dart_status dart_reduce_static(const dart_desc* desc, const void* X, const void* crit,
                               int32_t crit_D, int64_t crit_ld, const int64_t* pos, void* Y,
                               int64_t* pos_out, int32_t* keep, int32_t* cu_keep,
                               int32_t* piv_out, float* S_out, void* stream);

/* Size of the built-in scratch buffer of dart_reduce_static (host arithmetic only). */
DART_API size_t dart_static_scratch_bytes(void);

/* dart_device_status for the last dart_reduce_static call on the current GPU. */
DART_API dart_status dart_device_status_static(const dart_desc* desc, void* stream);

/* One per-token tensor for dart_compact_sequences: rows of row_bytes bytes (a multiple of
 * 16), row r of src at src + r*src_ld_bytes, likewise dst; bases and strides multiples of
 * 16.  src has desc.X_rows rows; dst needs room for the shortened batch. */
typedef struct dart_row_tensor {
  const void* src;      /* DEVICE */
  void* dst;            /* DEVICE, must not overlap src */
  int64_t row_bytes;
  int64_t src_ld_bytes;
  int64_t dst_ld_bytes;
} dart_row_tensor;

/* (d) for whole sequences -- Appendix D: the layers after the step see the text tokens and
 * the retained vision tokens; the key/value rows cached by the layers before it shrink the
 * same way (Table 2, KV-cache column).  Needs desc.span_start.  Sequence b is rows
 * [seq_cu[b], seq_cu[b+1]) of every per-token tensor (seq_cu: DEVICE int32[B+1], from 0 to
 * desc.X_rows, non-decreasing) and must contain its span; keep as produced by dart_reduce /
 * dart_topk_keep for the same descriptor.  Outputs:
 *   seq_cu_out [B+1]  offsets of the shortened sequences (the cu_seqlens a variable-length
 *                     attention kernel takes): sequence b keeps its rows before the span,
 *                     then rows span_start[b] + keep[.] in ascending order, then its rows
 *                     after the span;
 *   row_map [X_rows - total_N + sum of K_b at most]  row_map[r] = the row of the original
 *                     tensors that row r of the shortened batch is a copy of;
 *   tensors[i].dst    the n_tensors (HOST array, may be 0) tensors gathered by row_map, bit
 *                     copies (hidden states, per-layer key and value rows, ...);
 *   pos_out           pos_planes planes of position ids (plane p at pos + p*pos_plane_stride,
 *                     X_rows entries; e.g. 3 planes for multimodal rotary embeddings),
 *                     gathered into pos_out + p*pos_out_plane_stride; pos_planes may be 0.
 * A seq_cu that is not as described, or a span outside its sequence, sets every entry of
 * seq_cu_out to 0, copies nothing and makes dart_device_status report DART_ERR_DEVICE. */
DART_API dart_status dart_compact_sequences(const dart_desc* desc, const int32_t* seq_cu,
                                   const int32_t* keep, int32_t n_tensors,
                                   const dart_row_tensor* tensors, const int64_t* pos,
                                   int32_t pos_planes, int64_t pos_plane_stride, int64_t* pos_out,
                                   int64_t pos_out_plane_stride, int32_t* seq_cu_out,
                                   int32_t* row_map, void* ws, size_t ws_bytes, void* stream);

/* dart_reduce that also stamps the caller's HIP events with the begin and end of its
 * kernels: events is a HOST array of 12 hipEvent_t (as void*, created with timing enabled);
 * events[2k] takes the begin of the first kernel of stage k and events[2k+1] the end of its
 * last kernel (0 row norms, 1 pivot selection, 2 scores, 3 score ordering, 4 retained set,
 * 5 compaction), so hipEventElapsedTime(events[2k], events[2k+1]) is the stage's duration as
 * a kernel trace shows it: the times are the dispatches' own and nothing is enqueued between
 * the kernels.  A stage that launches no kernel for this descriptor (e.g. the ordering under
 * the single-threshold rule, the gather with Y == NULL) leaves its two events untouched.
 * The one-launch path (DART_FUSED=1) is not taken. */
DART_API dart_status dart_reduce_profiled(const dart_desc* desc, const void* X, const void* crit,
                                 int32_t crit_D, int64_t crit_ld, const int64_t* pos, void* Y,
                                 int64_t* pos_out, int32_t* keep, int32_t* cu_keep,
                                 int32_t* piv_out, float* S_out, void* ws, size_t ws_bytes,
                                 void* stream, void* const* events);

/* Waits for `stream`, then reports DART_ERR_DEVICE if the last call that used
 * `ws` (with this descriptor) skipped a ragged sample or met an invalid given pivot
 * list, DART_OK otherwise.  Every entry point that takes `ws` leaves these flags defined:
 * with DART_PIVOT_GIVEN, dart_reduce, dart_duplication_scores and dart_topk_keep validate the
 * piv array they read; an entry point that reads no pivots clears the pivot flag. */
DART_API dart_status dart_device_status(const dart_desc* desc, const void* ws, void* stream);

/* The absolute bound on |fp32 score - exact score| that dart_topk_keep and
 * dart_reduce certify decisions against, for this dtype. */
DART_API double dart_score_tolerance(int32_t dtype);

/* Diagnostic: the raw 32-term sums of the matrix-core instruction the bf16 score path is built
 * on (v_mfma_f32_16x16x32_bf16 from a zero accumulator).  A, B: DEVICE bf16 [tiles][16][32]
 * (k contiguous), out: DEVICE float [tiles][16][16], out[t][i][j] = sum_k A[t][i][k] *
 * B[t][j][k] as the hardware rounds it.  The bound of dart_score_tolerance assumes that this
 * sum errs by at most 16 * 2^-24 * sum_k |A B| (the instruction's internal rounding is not
 * documented); the test-suite checks that assumption through this call on the GPU it runs
 * on.  tiles >= 0; A, B, out 16-byte aligned. */
DART_API dart_status dart_probe_mfma_dot32(const void* A, const void* B, float* out,
                                           int32_t tiles, void* stream);

/* ---- attention on either side of the step -------------------------------------------------
 * The layers around the reduction step make the key rows whose norm step (a) ranks, and read the
 * rows that are left after step (d).  The calls below are that part of a layer: queries and
 * keys are normed and rotated by their position ids (which after the step are the carried ids
 * of the retained tokens, in one or several planes), keys and values go to a paged cache, and
 * attention reads the cache, for one new token of every sequence as for whole prompts.
 * Memory, streams, errors and determinism are as described at the top of this file; what is
 * checked on the device is reported in *status (see dart_cache).  Value range: any; infinities and
 * NaN in a row that is seen go into the results they belong to and no others, and what lies in
 * a page outside the keys of its sequence is never used.                                     */

/* How the heads of a layer are normed and rotated (host memory, plain data).
 * Element i of a head is x_i; with a weight, x is first replaced by
 *   x_i * weight_i / sqrt(mean_j x_j^2 + eps).
 * Pair p < rot/2 of a head, elements (p, p + rot/2), or (2p, 2p + 1) with interleaved, is then
 * turned by theta = position * inv_freq[p] (the angle in 64 bits, its sine and cosine in 32):
 *   (a, b) -> scale * (a cos - b sin, b cos + a sin);
 * elements from rot on pass.  All in 32 bits, rounded once to the type of the rows.          */
typedef struct dart_rotation {
  int32_t Hq;          /* query heads of a row, a multiple of Hkv, <= 1024                   */
  int32_t Hkv;         /* key heads (and value heads), >= 1                                  */
  int32_t d;           /* elements of a head: a multiple of 8, <= 256                         */
  int32_t dtype;       /* dart_dtype of rows, weights, outputs and pages                     */
  int32_t rot;         /* elements of a head that are turned: a multiple of 8, 0..d          */
  int32_t interleaved; /* 0: pairs (p, p + rot/2); 1: pairs (2p, 2p + 1)                     */
  int32_t planes;      /* planes of position ids, 1..4                                       */
  int32_t sections[4]; /* the first sections[0] pairs follow plane 0, the next sections[1]
                          plane 1, ...; they sum to rot/2 (ignored when planes == 1)         */
  const float* inv_freq; /* DEVICE float[rot/2]                                              */
  const void* q_weight;  /* DEVICE [d], or NULL: queries are not normed                      */
  const void* k_weight;  /* DEVICE [d], or NULL: keys are not normed                         */
  float eps;             /* >= 0                                                             */
  float scale;           /* factor of the turned elements (1 for plain rotations)            */
} dart_rotation;

/* Keys and values in pages, and the tokens of one call (host memory, plain data).  Key head h of
 * row r of page p is the d elements from p*page_ld + h*head_ld + r*row_ld of the key pool, the value
 * head likewise in the value pool; so pages may hold heads of rows (head_ld = page_size*row_ld) or
 * rows of heads (row_ld = Hkv*head_ld), and one page as long as a sequence is a plain cache.
 * Key j of sequence b is row j % page_size of page pages[b*pages_ld + j/page_size].
 * Tokens are packed: sequence b owns tokens cu_q[b] .. cu_q[b+1]-1 of the call, and kv_len[b] keys
 * of its own in the cache with this call's: its last n_b = cu_q[b+1] - cu_q[b] keys belong to
 * the call's tokens, in order (dart_attend without `causal` does not ask for that).
 * Shared prefixes (groups > 0): sequences group_cu[g] .. group_cu[g+1]-1 all see, before their own
 * keys, the prefix_len[g] keys of the pages prefix_pages[g*prefix_ld + ...], which are stored
 * once for all of them.
 * max_kv and max_prefix bound what the device arrays may hold, and divide the work: far above the lengths they cost time.
 * A sequence whose offsets decrease or leave 0..T, with more than max_q tokens, whose kv_len is below 0
 * or over max_kv or over pages_n*page_size, or whose prefix is as wrong, is skipped: nothing is appended
 * for it and its output is as if it saw no key; bit 0 of *status is set.  A page number outside
 * 0..n_pages-1 where a key is needed sets bit 1: the key is not appended, or the sequence's
 * output is unspecified.  status (DEVICE int32, or NULL) is only ever OR-ed into: the caller
 * clears it.                                                                                  */
typedef struct dart_cache {
  int32_t B;        /* sequences, 0..2^20 (0: the call writes nothing)                        */
  int32_t Hq, Hkv;  /* query heads, key/value heads: as dart_rotation                         */
  int32_t d;        /* elements of a head: a multiple of 8, <= 256                            */
  int32_t dtype;    /* dart_dtype of q, k, v, pools and out                                   */
  int32_t T;        /* tokens of the call, 0..2^24                                            */
  int32_t max_q;    /* host-known upper bound of every n_b                                    */
  int32_t max_kv;   /* host-known upper bound of every kv_len, 0..2^27                        */
  const int32_t* cu_q;   /* DEVICE int32[B+1] from 0 to T, or NULL: one token each (T == B)   */
  const int32_t* kv_len; /* DEVICE int32[B]                                                   */
  const int32_t* pages;  /* DEVICE int32[B][pages_ld]                                         */
  int32_t pages_ld;      /* entries from a row of `pages` to the next, >= 1                   */
  int32_t n_pages;       /* pages of the pools, >= 1                                          */
  int32_t page_size;     /* rows of a page: a power of two, 1..2^20                           */
  int64_t page_ld, head_ld, row_ld; /* strides in elements: multiples of 8 (of 4 for 32-bit rows), d <= row_ld,
                                       0 <= head_ld, 0 <= page_ld, none over 2^33             */
  int32_t groups;     /* shared prefixes, 0..B (0: none, the fields below are ignored)        */
  int32_t max_prefix; /* host-known upper bound of every prefix_len, 0..2^27                  */
  const int32_t* group_cu;     /* DEVICE int32[groups+1] from 0 to B                          */
  const int32_t* prefix_pages; /* DEVICE int32[groups][prefix_ld]                             */
  const int32_t* prefix_len;   /* DEVICE int32[groups]                                        */
  int32_t prefix_ld;           /* entries from a row of `prefix_pages` to the next, >= 1      */
  int32_t pages_n;             /* entries of a row of `pages`, where the table is a view of a wider one; 0: pages_ld.  No
                                  entry past them is read                                     */
  int32_t prefix_n;            /* the same of `prefix_pages`; 0: prefix_ld                    */
} dart_cache;

/* Norms and rotates the heads of T tokens: head h of token t of q is the d elements from t*q_ld + h*d,
 * of k from t*k_ld + h*d (so both may be views of a fused projection's rows); outputs likewise, and
 * q_out may be q, k_out may be k.  Bases and strides are multiples of 16 bytes.
 * pos: position ids, plane p of token t at pos[p*pos_plane_stride + t]; any value.  The stride is at least T, or 0: one plane
 * stands for all.
 * l1_out (optional, float[T]): the L1 norm of every key row as it is stored (all Hkv heads, after
 * rounding): the criterion norms that dart_reduce_with_norms takes with k_out as the criterion
 * rows, good to 2^-20 of their value.                                                         */
DART_API dart_status dart_norm_rotate(const dart_rotation* rotation, int32_t T, const void* q,
                                      int64_t q_ld, const void* k, int64_t k_ld, const int64_t* pos,
                                      int64_t pos_plane_stride, void* q_out, int64_t q_out_ld,
                                      void* k_out, int64_t k_out_ld, float* l1_out, void* stream);

/* The same for the tokens of `cache`, whose keys go to their pages, and with them the values (v, laid
 * out like k, copied): token i of sequence b becomes key kv_len[b] - n_b + i, so kv_len[b] >= n_b is
 * required.  k_out is optional here (rows of the keys beside the pages); k_out_ld is ignored without it.
 * The queries of tokens that are not appended are written all the same.  Pages that two tokens of
 * a call name as the same row get either's.                                                   */
DART_API dart_status dart_norm_rotate_append(const dart_rotation* rotation, const dart_cache* cache,
                                             const void* q, int64_t q_ld, const void* k, int64_t k_ld,
                                             const void* v, int64_t v_ld, const int64_t* pos,
                                             int64_t pos_plane_stride, void* q_out, int64_t q_out_ld,
                                             void* k_out, int64_t k_out_ld, float* l1_out, void* k_pool,
                                             void* v_pool, int32_t* status, void* stream);

/* Bytes of workspace dart_attend needs for this descriptor (host arithmetic only; 0 if it is
 * invalid). */
DART_API size_t dart_attend_workspace_bytes(const dart_cache* cache);

/* Attention over the cache.  Query head h of token t (d elements from t*q_ld + h*d, read with key head
 * h / (Hq/Hkv)) sees its group's prefix and, of its sequence's own keys, those up to its own place:
 * token i of sequence b sees keys j <= kv_len[b] - n_b + i with `causal`, all kv_len[b] without.  With
 * s_j = scale * <q, k_j> and m the largest of them,
 *   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   lse = m + ln sum_j exp(s_j - m);
 * a token that sees nothing, or only scores of -infinity, gets zeros and -infinity; a token that no
 * sequence owns is not written.  out has the layout of q; lse (optional) is float[T][Hq].  Scores, sums and the running
 * result are held in 32 bits (a score as s_j * log2 e: what 32 bits do not hold of that is an infinity); with bfloat16 rows the
 * factors exp(s_j - m) are rounded to bfloat16 for the product with the values (and only there).
 * A prefix is read once for every tile of up to 256 (token, query head) pairs of a key head, not for every sequence of its group.
 * Heads are worked on as 64, 128 or 256 elements, whichever holds them.  scale is finite.
 * T * (Hq/Hkv) is at most 2^28, and T * Hq at most 2^24 where there are prefixes or the keys of few
 * tokens are divided over the chip (beyond: DART_ERR_SHAPE, and 0 bytes of workspace). */
DART_API dart_status dart_attend(const dart_cache* cache, const void* q, int64_t q_ld,
                                 const void* k_pool, const void* v_pool, float scale, int32_t causal,
                                 void* out, int64_t out_ld, float* lse, void* ws, size_t ws_bytes,
                                 int32_t* status, void* stream);

/* ---- a cache held in 4 bits -----------------------------------------------------------------
 * The same cache with a quarter of the bytes.  A head's row is cut into blocks of 32 values (the last one filled up
 * with zeros); a block is 32 codes of 4 bits and one byte e, its scale 2^(e - 127).  A code is a sign (bit 3) and one of
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bits 0-2: 0..7); the value is their product, which bfloat16 and 32 bits hold exactly.
 * e is the smallest from 0 to 252 that leaves the block's largest value under 7 * 2^(e - 127) (252: whatever it is), and a
 * value becomes the nearest of the 15, a tie the even code, the largest where it lies beyond.  A block with an infinity or
 * NaN has e = 255 and is read as NaN throughout.  No call writes 253 or 254; they are read as their products, infinities where
 * those pass the type's range.
 * A pool is two arrays: `codes` (16-byte aligned) and `scales`.  With W = d rounded up to 32, the strides page_ld, head_ld and
 * row_ld of its dart_cache count values and are multiples of 32, W <= row_ld: key head h of row r of page p has value i at bit
 * 4 * (x + i) of codes, x = p*page_ld + h*head_ld + r*row_ld (the even value of a byte in its low half), and the
 * scale of block j at scales[x / 32 + j].  dtype is that of the rows (k, v, q, out).  Everything else of dart_cache holds as
 * it stands there.                                                                            */

/* Writes key and value rows (laid out as in dart_norm_rotate_append, keys turned already) to their places in 4-bit pages:
 * token i of sequence b becomes key kv_len[b] - n_b + i, so kv_len[b] >= n_b is required.  A row of a page that two tokens of
 * a call name gets codes and scales of either. */
DART_API dart_status dart_append_4bit(const dart_cache* cache, const void* k, int64_t k_ld, const void* v, int64_t v_ld,
                                      void* k_codes, void* k_scales, void* v_codes, void* v_scales, int32_t* status,
                                      void* stream);

/* The other way: the rows of the call's tokens as the pages hold them (all keys of sequence b with n_b = kv_len[b]), e.g. as
 * the criterion rows of dart_reduce.  k_out or v_out may be NULL; their pools are then not looked at.  Rows of tokens that have
 * no key are left as they were. */
DART_API dart_status dart_read_4bit(const dart_cache* cache, const void* k_codes, const void* k_scales, const void* v_codes,
                                    const void* v_scales, void* k_out, int64_t k_ld, void* v_out, int64_t v_ld,
                                    int32_t* status, void* stream);

/* Bytes of workspace dart_attend_4bit needs for this descriptor (host arithmetic only; 0 if it is invalid). */
DART_API size_t dart_attend_4bit_workspace_bytes(const dart_cache* cache);

/* dart_attend with the keys and values that the codes stand for; numerics and limits are its own. */
DART_API dart_status dart_attend_4bit(const dart_cache* cache, const void* q, int64_t q_ld, const void* k_codes,
                                      const void* k_scales, const void* v_codes, const void* v_scales, float scale,
                                      int32_t causal, void* out, int64_t out_ld, float* lse, void* ws, size_t ws_bytes,
                                      int32_t* status, void* stream);

/* ---- eviction -------------------------------------------------------------------------------
 * A cache that grows with its answers is cut to the keys that attention uses: the weight of every key is gathered while the
 * answers are made, and from time to time the keys that gathered least are dropped, each key head choosing its own.
 * Weights are float[n_pages][Hkv][page_size], contiguous: that of key head h of row r of page p at
 * (p*Hkv + h)*page_size + r, so that the page table of the keys is theirs too.  Both calls take pools of rows
 * (k_scales and v_scales NULL) or held in 4 bits (codes and scales); `four_bit` says so where no pool is given.          */

/* Bytes of workspace dart_attend_weights needs for this descriptor (host arithmetic only; 0 if it is invalid). */
DART_API size_t dart_attend_weights_workspace_bytes(const dart_cache* cache, int32_t four_bit);

/* What the keys gather from the call's tokens.  For key j of a sequence (or of a group's prefix), per key head,
 *   w_j <- carry * w_j + sum exp(scale * <q, k_j> - lse)
 * over the (token, query head of the key head) pairs that see it, as dart_attend defines that; q, lse and causal as they went
 * to it or came from it.  Keys that belong to the call's tokens start from 0, whatever their weight was, and with carry 0
 * all do (what was there is not read).  A pair whose lse is -infinity gives nothing; another one that is no number, or
 * infinite, goes into the weights of the keys it sees, as the formula has it.  The weights of a sequence (or group) without
 * tokens, and of one that is skipped, are left as they were; a group with a sequence that is skipped is skipped.  A key that two
 * sequences (or a sequence and a prefix) of the call have gets what either gives.  Sums in 32 bits, in a fixed order; a
 * factor errs by some 2^-22 of its score's and lse's magnitude, beside what lse itself does.  scale and carry are finite.
 * max_kv, max_prefix and max_q choose the kernel and divide the work, whatever the lengths are: two prompts of 9216 tokens take
 * 705 us, 1735 with a max_kv of 131 072.  T * (Hq/Hkv) is at most 2^28, and B * Hkv times max_kv, groups * Hkv times max_prefix,
 * in tiles of the kernel's 128 to 512 keys, at most 2^30 (beyond: DART_ERR_SHAPE, and 0 bytes of workspace). */
DART_API dart_status dart_attend_weights(const dart_cache* cache, const void* q, int64_t q_ld, const void* k_pool,
                                         const void* k_scales, const float* lse, float scale, int32_t causal, float carry,
                                         float* weights, void* ws, size_t ws_bytes, int32_t* status, void* stream);

/* How many keys a sequence keeps (host memory, plain data): of kv keys
 *   min(kv, max(K, first + recent)),   K = budget, or floor(kv * ratio_num / ratio_den) where budget is 0. */
typedef struct dart_eviction {
  int32_t budget;    /* 0..: keys, or 0: the ratio counts                                     */
  int32_t ratio_num; /* 0..ratio_den                                                          */
  int32_t ratio_den; /* >= 1 where it counts                                                  */
  int32_t first;     /* keys at the front that are always kept, 0..2^27                       */
  int32_t recent;    /* keys at the end that are always kept, 0..2^27                         */
} dart_eviction;

/* The most keys that a sequence of max_kv keeps: the entries that a row of `kept` needs (-1: invalid). */
DART_API int32_t dart_evict_most(const dart_cache* cache, const dart_eviction* eviction, int32_t four_bit);

/* Bytes of workspace dart_evict needs (host arithmetic only; 0 if a descriptor is invalid): 4 for each key that may be kept, by
 * max_kv, whether `kept` is given or not. */
DART_API size_t dart_evict_workspace_bytes(const dart_cache* cache, const dart_eviction* eviction, int32_t four_bit);

/* Cuts every sequence of the cache: each key head keeps the first and the recent keys, and of those between the ones of largest
 * weight, of equals the first; NaN counts as less than any weight.  Kept keys keep their order and move, in place, to the
 * front of the sequence's pages, values with them.  What lies behind them is unspecified, the pages there are free.
 *   weights_out  optional, laid out like weights and may be weights: the kept keys' weights, moved like them
 *   kept         optional, int32 [B][Hkv] rows kept_ld apart: the places that the kept keys had, ascending
 *   kv_len_out   int32 [B]: keys of each sequence after the call; may be the array that cache->kv_len names
 * The tokens of the descriptor (T, cu_q, max_q) and its groups play no part beyond its being a valid one; to cut prefixes describe
 * them as sequences.  max_kv chooses the kernel, whatever the lengths are (637 keys 13 us, 21 with a bound of 16 384).  A
 * sequence whose kv_len is below 0 or over max_kv or its pages is skipped and bit 0 of *status set.  Keys in pages outside 0..n_pages-1
 * count as less than any weight and are not moved, and bit 1 is set.  Pages that are named twice for keys of this call, by one
 * sequence or by two, hold unspecified rows afterwards unless all of them keep all keys.  B * Hkv times the
 * keys kept is at most 2^40. */
DART_API dart_status dart_evict(const dart_cache* cache, const dart_eviction* eviction, void* k_pool, void* k_scales,
                                void* v_pool, void* v_scales, const float* weights, float* weights_out, int32_t* kept,
                                int64_t kept_ld, int32_t* kv_len_out, void* ws, size_t ws_bytes, int32_t* status,
                                void* stream);

/* Static, NUL-terminated description of a status code. */
DART_API const char* dart_strerror(dart_status status);

#ifdef __cplusplus
}
#endif
#endif /* DART_H_ */
