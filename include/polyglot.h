/*
 * polyglot.h -- C ABI of the MI355X (gfx950) library for the minibatch SGD
 * step of the Polyglot window-ranking language model.
 *
 * Method.  Kulkarni, Al-Rfou, Perozzi, Skiena, "Exploring the power of GPU's
 * for training Polyglot language models" (arXiv:1404.1521).  The paper trains
 * the Polyglot model, a SENNA-like ranking language model (§1 Introduction),
 * with minibatch SGD (batch size discussion, §4.6), and finds that the
 * embedding-gradient update -- the "advanced indexing" increment that adds
 * row k of Y to row I[k] of W for every k (§4.2, Table 1:
 * GpuAdvancedIncSubtensor1) -- dominates training time; §4.3 replaces it
 * with a parallel kernel.  The paper does not write the model out; this
 * library implements the SENNA-style window ranker:
 *
 *   x     = concat(E[w_0] .. E[w_{win-1}])          K = win*d values
 *   x~    = x with block c = win/2 replaced by E[corrupt]
 *   s(x)  = w2 . tanh(W1 x + b1) + b2
 *   loss  = (1/B) sum_b max(0, 1 - s(x_b) + s(x~_b))
 *
 * and one SGD step P <- P - lr * dloss/dP over E, W1, b1, w2, b2, all
 * gradients taken at the pre-step parameters.  The hinge derivative at a
 * margin of exactly 0 is taken as 0.  A corrupt id equal to the true centre
 * is used as drawn (its gradient cancels).
 *
 * Conventions for every entry point.
 *   - All tensor arguments are DEVICE pointers (hipMalloc / torch CUDA
 *     tensors on the device the context was created on), C-contiguous,
 *     row-major, float32 or int32, owned by the caller.  The library never
 *     frees or retains them after the call returns.
 *   - Work is enqueued asynchronously on the context's HIP stream; the
 *     caller must synchronise that stream before reading results on the
 *     host or touching the buffers from another stream.
 *   - Return value: POLYGLOT_OK (0) or a negative POLYGLOT_E* code.  Errors
 *     that the host can detect (bad sizes, NULL pointers, non-finite lr,
 *     batch above the configured maximum) are returned before anything is
 *     enqueued.  Ids outside [0, V) are detected on the device: the step
 *     then modifies no parameter, writes NaN to its loss slot, and raises a
 *     sticky flag that polyglot_status() reports as POLYGLOT_EID.
 *   - A context is not thread-safe and must be used from one host thread
 *     and one stream at a time.
 *
 * Layouts (int32 ids, float32 values):
 *   E[V][d]  W1[H][win*d]  b1[H]  w2[H]  b2[1]
 *   windows[B][win] (centre at win/2)  corrupt[B]
 */
#ifndef POLYGLOT_H
#define POLYGLOT_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define POLYGLOT_OK 0
#define POLYGLOT_EINVAL -1 /* bad dimension, even window, non-finite lr, bad mode */
#define POLYGLOT_ENULL -2  /* a required pointer is NULL */
#define POLYGLOT_EBATCH -3 /* B or N <= 0, or above the context's maximum */
#define POLYGLOT_EHIP -4   /* HIP runtime error; text in polyglot_last_error() */
#define POLYGLOT_EID -5    /* an id was outside [0, V) (reported by polyglot_status) */
#define POLYGLOT_ESTATE -6 /* call not valid in the context's current state */
#define POLYGLOT_EOFFSETS -7 /* sequence offsets did not ascend from 0 to the token count
                                (reported by polyglot_status) */

/* How the embedding-gradient rows are added into the table (§4.3). */
#define POLYGLOT_SCATTER_SORTED 0 /* stable radix sort by row id, segmented sum: deterministic */
#define POLYGLOT_SCATTER_ATOMIC 1 /* one float atomic add per (entry, column): order-dependent rounding */

typedef struct polyglot_ctx polyglot_ctx;

typedef struct {
  int32_t V;            /* vocabulary rows of E, >= 1 */
  int32_t d;            /* embedding width, multiple of 16, 16..256; for H <= 64,
                           W1 (H x win*d floats) must also fit one workgroup's LDS */
  int32_t win;          /* window length, odd, 1..31 */
  int32_t H;            /* hidden units: 1..64, or a multiple of 64 up to 256 with d a
                           multiple of 64 (wide layers run as three separate
                           contractions: forward, dW1, per-entry gradient rows) */
  int32_t max_batch;    /* largest B accepted by train_step / score / gather */
  int32_t scatter_mode; /* POLYGLOT_SCATTER_SORTED or POLYGLOT_SCATTER_ATOMIC */
  int32_t max_scatter;  /* largest N accepted by polyglot_scatter_add (0: no workspace) */
  int32_t max_rows;     /* largest table row count for polyglot_scatter_add */
} polyglot_config;

/* Creates a context on the current HIP device.  `stream` is a hipStream_t
 * (NULL = the legacy default stream).  All workspace is allocated here, once,
 * sized for cfg->max_batch and cfg->max_scatter; of the calls below only
 * polyglot_reserve_recurrence and polyglot_reserve_logits allocate more.
 * On success *out receives the context; on error *out is left NULL. */
int polyglot_init(const polyglot_config* cfg, void* stream, polyglot_ctx** out);

/* Waits for the context's stream, frees its workspace and the context. */
int polyglot_destroy(polyglot_ctx* ctx);

/* Replaces the stream the context enqueues on (hipStream_t, NULL = default).
 * All calls of a context share its workspace and must run one after the other.
 * What is enqueued after the change therefore waits for what the old stream holds
 * (an event; if the old stream no longer exists, for the device).  That leaves the
 * calls that a graph capture records: where either stream is capturing nothing is
 * ordered, and the program sees to it that a graph's replay overlaps neither
 * another replay nor a call of the same context on another stream.  Calls that
 * overlap all the same may leave outputs unwritten.  Where the sequence operators
 * notice it, polyglot_status returns POLYGLOT_EHIP; their workspace is then to be
 * reserved again. */
int polyglot_set_stream(polyglot_ctx* ctx, void* stream);

/* One SGD step of the window-ranking model (model above; the embedding
 * update is the row scatter-add of §4.2/§4.3), in place on E, W1, b1, w2,
 * b2.  windows[B][win] and corrupt[B] are int32 ids in [0, V).  lr is the
 * SGD learning rate.  loss_dev, if not NULL, is a device float that
 * receives the mean hinge loss at the pre-step parameters (NaN if an id was
 * out of range).  1 <= B <= max_batch. */
int polyglot_train_step(polyglot_ctx* ctx, float* E, float* W1, float* b1, float* w2, float* b2,
                        const int32_t* windows, const int32_t* corrupt, int32_t B, float lr,
                        float* loss_dev);

/* polyglot_train_step followed by a synchronisation: the step is enqueued on
 * the context's stream with its loss in a library-owned device slot, the
 * stream is synchronised, and the mean hinge loss (the quantity of the
 * model above, at the pre-step parameters) is written to *loss_host (host
 * memory, caller-owned).  Returns what polyglot_train_step returns for the
 * arguments (nothing is enqueued on such an error and *loss_host is left
 * unchanged); POLYGLOT_EHIP if the synchronisation fails; POLYGLOT_EID (or
 * POLYGLOT_EOFFSETS, left by a sequence operator) if a device error word is raised
 * once the step has run, in which case the step changed no parameter and
 * *loss_host is NaN.  The error words stay raised
 * (every later step is void) until polyglot_status() clears them. */
int polyglot_train_step_sync(polyglot_ctx* ctx, float* E, float* W1, float* b1, float* w2,
                             float* b2, const int32_t* windows, const int32_t* corrupt,
                             int32_t B, float lr, float* loss_host);

/* S consecutive SGD steps, step s using windows + s*B*win and corrupt + s*B,
 * exactly as S calls of polyglot_train_step.  losses_dev[S] (device, may be
 * NULL) receives each step's loss.  The launches of the S steps are recorded
 * once into a HIP graph that the context caches (keyed on every argument)
 * and replays, which removes per-kernel host launch cost. */
int polyglot_train_steps(polyglot_ctx* ctx, float* E, float* W1, float* b1, float* w2,
                         float* b2, const int32_t* windows, const int32_t* corrupt, int32_t S,
                         int32_t B, float lr, float* losses_dev);

/* The score of the ranking model of §1 Introduction (the SENNA-like
 * network the paper trains), s(x) = w2 . tanh(W1 x + b1) + b2, of each of
 * the B windows: x = concat_j E[windows[b][j]].  windows[B][win] int32
 * (device), scores_dev[B] float32 (device, written).  A window holding an
 * out-of-range id scores NaN and raises the sticky flag.  1 <= B <= max_batch;
 * E and W1 16-byte aligned (else POLYGLOT_EINVAL). */
int polyglot_score(polyglot_ctx* ctx, const float* E, const float* W1, const float* b1,
                   const float* w2, const float* b2, const int32_t* windows, int32_t B,
                   float* scores_dev);

/* The window gather on its own: the input vector x of the §1 Introduction
 * model, the concatenation of the window's embedding rows, for every
 * window, X[B][win*d] = concat_j E[windows[b][j]], and the corrupted centre
 * rows Xc[B][d] = E[corrupt[b]] (bit-exact copies; a row with an
 * out-of-range id is written as NaN and raises the sticky flag).  All
 * pointers device; E, X and Xc 16-byte aligned; 1 <= B <= max_batch. */
int polyglot_gather(polyglot_ctx* ctx, const float* E, const int32_t* windows,
                    const int32_t* corrupt, int32_t B, float* X, float* Xc);

/* The advanced-indexing increment of §4.2/§4.3: for every k in [0, N),
 * table[idx[k]] += alpha * Y[k], where repeated indices accumulate.
 * table[rows][d], idx[N] int32 in [0, rows), Y[N][d].  mode selects the
 * sorted-segment or the atomic algorithm.  N <= max_scatter,
 * rows <= max_rows, d a multiple of 4 up to 256.  Out-of-range indices
 * leave the table untouched and raise the sticky flag. */
int polyglot_scatter_add(polyglot_ctx* ctx, float* table, int32_t rows, int32_t d,
                         const int32_t* idx, const float* Y, int32_t N, float alpha,
                         int32_t mode);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the sorted
 * mode of polyglot_scatter_add -- table[idx[k]] += alpha * Y[k] for every k in
 * [0, N), repeated indices accumulated in entry order, each touched row
 * written once -- with no context.  It allocates nothing: its sort buffers
 * live in a static device array of POLYGLOT_NOALLOC_SCRATCH_BYTES that the
 * library holds on every GPU it runs on until the process ends.
 *   table[rows][d], Y[N][d] float32 and idx[N] int32: device pointers owned by
 *     the caller; table and Y 16-byte aligned; d a multiple of 4 up to 256;
 *     1 <= rows <= POLYGLOT_NOALLOC_MAX_ROWS.
 *   1 <= N <= POLYGLOT_NOALLOC_MAX_N, else POLYGLOT_EBATCH.
 *   status_dev: device int32 (may be NULL), written on the device with
 *     POLYGLOT_OK, or POLYGLOT_EID when an index is outside [0, rows), in
 *     which case the call leaves the table untouched.  Nothing is sticky:
 *     every call starts clean.
 *   stream: hipStream_t the two launches go on (NULL = the default stream).
 * Returns POLYGLOT_OK once enqueued, POLYGLOT_ENULL, POLYGLOT_EBATCH,
 * POLYGLOT_EINVAL (rows, d, alignment, non-finite alpha) before anything is
 * enqueued, or POLYGLOT_EHIP.  All calls on one GPU share its scratch array:
 * calls that may overlap in time on one GPU (several streams or host
 * threads) race and must be serialised by the caller. */
#define POLYGLOT_NOALLOC_MAX_N 8192
#define POLYGLOT_NOALLOC_MAX_ROWS (1 << 26)
#define POLYGLOT_NOALLOC_SCRATCH_BYTES 66816
int polyglot_scatter_add_noalloc(float* table, int32_t rows, int32_t d, const int32_t* idx,
                                 const float* Y, int32_t N, float alpha, int32_t* status_dev,
                                 void* stream);

/* Storage formats and operations of polyglot_scatter_update. */
#define POLYGLOT_F32 0  /* IEEE binary32 */
#define POLYGLOT_BF16 1 /* bfloat16: the upper 16 bits of a binary32 */
#define POLYGLOT_F16 2  /* IEEE binary16 */
#define POLYGLOT_OP_INC 0 /* table[idx[k]] += alpha * Y[k] */
#define POLYGLOT_OP_SET 1 /* table[idx[k]] = Y[k]; alpha unused */

/* The general advanced-indexing op of §4.3 (the increment the paper
 * rewrites, in the library form it contributes: any table format, any
 * index vector, increment or assignment).
 *   table[rows][d] and Y[N][d]: device, row-major, both in storage format
 *     dtype; d in [1, 256]; aligned to their element size.
 *   idx[N]: device, int32 (idx_bytes 4) or int64 (idx_bytes 8), each in
 *     [0, rows); aligned to idx_bytes.
 *   op POLYGLOT_OP_INC: for every k, table[idx[k]] += alpha * Y[k];
 *     repeated indices accumulate.  Sorted mode adds each row's entries in
 *     float32 in entry order and rounds the row to its format once (round
 *     to nearest even).  Atomic mode: float32 tables only, one float atomic
 *     per element.
 *   op POLYGLOT_OP_SET: for every k in order, table[idx[k]] = Y[k]; for a
 *     repeated index the largest k wins (sorted mode only).
 * N <= max_scatter and rows <= max_rows of the context.  Float32 increments
 * take the same kernels as polyglot_scatter_add.  Faster forms, with the
 * same results: 16-bit increments whose rows are whole 4-byte words (d even,
 * table and Y 4-byte aligned) read and write two rows per word; assignments
 * copy rows in the widest words (up to 16 bytes) that divide a row and both
 * pointers' alignment.  The caller owns every
 * buffer; the call is asynchronous on the context stream.  Returns
 * POLYGLOT_EINVAL for a bad format, op, mode, width or alignment or an
 * unsupported mode combination, POLYGLOT_ENULL, POLYGLOT_EBATCH; an index
 * outside [0, rows) leaves the table untouched and raises the sticky flag
 * (POLYGLOT_EID from polyglot_status). */
int polyglot_scatter_update(polyglot_ctx* ctx, void* table, int32_t dtype, int32_t rows,
                            int32_t d, const void* idx, int32_t idx_bytes, const void* Y,
                            int32_t N, float alpha, int32_t op, int32_t mode);

/* The distinct values of the index vector I of the §4.2 increment
 * W[I[k]] += Y[k] in the last sorted-mode train step: the rows of E the step
 * updated (ids of the windows and the corrupt ids), ascending.  Synchronises
 * the stream.  ids_host: host array of cap ints (may be NULL with cap 0);
 * at most cap ids are written and the total to *count (host).
 * POLYGLOT_ESTATE if no sorted-mode step has run, or if a scatter-add has
 * reused the sort buffers since. */
int polyglot_touched_rows(polyglot_ctx* ctx, int32_t* ids_host, int32_t cap, int32_t* count);

/* Kernel ids reported by polyglot_kernel_times. */
#define POLYGLOT_K_FWDBWD 0   /* fused gather + forward + hinge + backward (+ sort start);
                                 wide layers: gather + forward + hinge + per-window dz */
#define POLYGLOT_K_SORT 1     /* entry sort launches of a step (large batches) or of
                                 polyglot_scatter_add */
#define POLYGLOT_K_UPDATE 2   /* embedding segmented update + dense SGD */
#define POLYGLOT_K_GATHER 3   /* polyglot_gather */
#define POLYGLOT_K_SCATTER 4  /* polyglot_scatter_add's table update (atomic mode: and the id
                                 check); its sort and fix-up count under SORT and SEGFIX */
#define POLYGLOT_K_SCORE 5    /* polyglot_score */
#define POLYGLOT_K_SEGFIX 6   /* rows whose sorted entries span several chunks */
#define POLYGLOT_K_WIDE_DW1 7 /* wide layers: dW1 partials over window slices */
#define POLYGLOT_K_WIDE_G 8   /* wide layers: per-entry embedding gradient rows */
#define POLYGLOT_NKERNELS 9

/* Per-kernel timing for measurement.  With enable != 0 every later kernel
 * launch of this context (outside graph capture) gets a start/stop event
 * pair that the HIP runtime binds to the kernel's own dispatch
 * (hipExtLaunchKernel), so the elapsed time is the kernel's execution, not
 * the host enqueue.  polyglot_kernel_times() synchronises the streams,
 * writes the summed elapsed milliseconds and the launch count of each kernel
 * id into ms[POLYGLOT_NKERNELS] and launches[POLYGLOT_NKERNELS] (host
 * arrays), and resets the sums.  An id with several launches in one call
 * (the sort: histogram and radix passes) sums all of them. */
int polyglot_set_timing(polyglot_ctx* ctx, int enable);
int polyglot_kernel_times(polyglot_ctx* ctx, double* ms, int32_t* launches);

/* ------------------------------------------------------------------ sequences
 * Operators of a language model that reads all of its context and not a
 * window of it, over the same word table: rows gathered with dropout, a gated
 * linear recurrence over packed sequences, and the choice of a word among a
 * vocabulary's scores.  They need a context for its stream, its error words
 * and its workspace; the context's model shape does not matter to them.
 *
 * Common to all: tensors are device pointers owned by the caller, in the
 * storage format `dtype` (POLYGLOT_F32, POLYGLOT_BF16, POLYGLOT_F16) unless a
 * type is stated, aligned to their element size, with rows of consecutive
 * elements; ld_* is the distance between rows in elements, at least a row's
 * length.  Element offsets may pass 2^32.  Arithmetic, sums and states are in
 * 32 bits; each output is rounded to its format once (to nearest even).  Calls
 * are asynchronous on the context's stream and may be captured into a HIP
 * graph, whose replays must not overlap each other or the context's other calls
 * (polyglot_set_stream).  The argument blocks are read before the call returns; fields that
 * are not set must be zero.  Results do not depend on strides or alignment.
 * Host-detectable errors: POLYGLOT_ENULL, POLYGLOT_EINVAL,
 * POLYGLOT_EBATCH (above the reserved workspace), nothing enqueued. */

/* Dropout with a mask that is computed and never stored.
 *
 *   y[r][c] = keep(r, c) ? x[r][c] / (1 - p') : 0,   plus add[r][c] if add
 *
 * keep(r, c) compares 16 random bits with t = round(65536 p); p' = t / 65536.
 * The bits are piece c % 8 (low half of a word first) of the four words that
 * Philox 4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy
 * as 1, 2, 3", SC 2011) gives for the counter
 *   {c / 8, low and high word of first_row + r, site + *site_dev}
 * and the key `seed` (low word first).  They depend on nothing else: not on the
 * format, the strides, or how rows are divided among calls.  The gradient of y
 * with respect to x is the same operator on dy with the same seed, site and
 * first_row (and no add); that of add is dy itself.
 *   whole_rows != 0: a row is kept or dropped as a whole, by piece 0 at c / 8 = 2^32 - 1.
 *   ids != NULL: row r of x is row ids[r] of a table x[table_rows][d].  An id
 *     outside the table makes its row NaN (as in polyglot_gather) and raises the
 *     sticky flag (POLYGLOT_EID).
 * A dropped element is exactly 0 (plus add) also where x is not finite; p = 0
 * copies, p = 1 drops everything.  y may be x (without ids) or add, with the same
 * ld.  rows = 0 does nothing. */
typedef struct {
  const void* x;
  const void* add; /* [rows][d] or NULL */
  void* y;         /* [rows][d] */
  const void* ids; /* [rows] int32 or int64, or NULL */
  const uint32_t* site_dev; /* device word added to site (a step counter of a captured
                               graph), or NULL */
  int64_t rows, ld_x, ld_add, ld_y;
  uint64_t seed, first_row;
  uint32_t site;      /* which dropout of which step */
  float p;            /* in [0, 1] */
  int32_t d;          /* >= 1 */
  int32_t dtype;
  int32_t id_bytes;   /* 4 or 8 with ids */
  int32_t table_rows; /* >= 1 with ids */
  int32_t whole_rows;
} polyglot_dropout_args;
int polyglot_dropout(polyglot_ctx* ctx, const polyglot_dropout_args* args);

/* Gated linear recurrence over packed sequences.
 *
 *   POLYGLOT_GATE_RAW:      h_t = a_t h_{t-1} + x_t             a = gate
 *   POLYGLOT_GATE_SIGMOID:  h_t = a_t h_{t-1} + (1 - a_t) x_t   a = 1 / (1 + e^-gate)
 *
 * for each of D channels on its own; `group` consecutive channels share a gate
 * (a head), so gate has D / group columns.  Sequence s is the tokens
 * [offsets[s], offsets[s+1]); without offsets all nseq sequences have
 * tokens / nseq tokens.  Sequences may be empty.  h_{-1} is h0[s] (zeros if
 * NULL); last[s], if not NULL, receives the state after the sequence's last
 * token (h0[s] or zeros for an empty one); last may be h0.  reverse != 0 reads
 * every sequence from its last token to its first.  The state is carried in
 * 32 bits from the sequence's start to its end; h holds its roundings to dtype.
 * h may be x, with the same ld.  Consecutive gates are multiplied with each other:
 * RAW gates above 1 in size over many tokens may take such a product past 32 bits'
 * range, and the state with it, where one token after the other would not.  What is
 * infinite, a state or a RAW gate, may come out as NaN further on in its sequence and
 * channel where one token after the other would keep it infinite.
 * Widths (with shared gates: groups) of whole fours of channels are the fast ones.
 *
 * With one token per sequence (tokens == nseq, no offsets) this is a model's
 * step for single tokens: one pass over the rows, no workspace.  Other calls
 * use the workspace of polyglot_reserve_recurrence.
 * Offsets that do not ascend from 0 to `tokens` raise POLYGLOT_EOFFSETS
 * (polyglot_status); the outputs are then unspecified, and no access leaves
 * the tensors. */
#define POLYGLOT_GATE_RAW 0
#define POLYGLOT_GATE_SIGMOID 1
typedef struct {
  const void* gate;    /* [tokens][D / group] */
  const void* x;       /* [tokens][D] */
  const float* h0;     /* [nseq][D] or NULL */
  const void* offsets; /* [nseq + 1] int32 or int64, or NULL */
  void* h;             /* [tokens][D] */
  float* last;         /* [nseq][D] or NULL */
  int64_t tokens;      /* 0 .. 2^31 - 1 */
  int64_t ld_gate, ld_x, ld_h;
  int32_t nseq;         /* >= 1 */
  int32_t D;            /* >= 1 */
  int32_t group;        /* 1, or 2..256 dividing D */
  int32_t dtype;
  int32_t offset_bytes; /* 4 or 8 with offsets */
  int32_t form;         /* POLYGLOT_GATE_* */
  int32_t reverse;
} polyglot_recurrence_args;
int polyglot_recurrence(polyglot_ctx* ctx, const polyglot_recurrence_args* args);

/* The gradient of polyglot_recurrence.  With dh the gradient of h and dlast that
 * of last, going from a sequence's last token to its first:
 *
 *   lambda_t = dh_t + mu_{t+1},  mu_t = a_t lambda_t  (mu after the last token: dlast[s])
 *   RAW:      dx_t = lambda_t             dgate_t = sum over the group of lambda_t h_{t-1}
 *   SIGMOID:  dx_t = (1 - a_t) lambda_t   dgate_t = a_t (1 - a_t) sum lambda_t (h_{t-1} - x_t)
 *   dh0[s] = mu of the sequence's first token (dlast[s] or zeros for an empty one)
 *
 * h is the forward call's output: h_{t-1} enters with its rounding to dtype.
 * x may be NULL for POLYGLOT_GATE_RAW.  dgate must not overlap an input; dx may
 * be dh or x, with the same ld.  dh0 may be dlast. */
typedef struct {
  const void* gate;    /* [tokens][D / group] */
  const void* x;       /* [tokens][D] */
  const void* h;       /* [tokens][D] */
  const void* dh;      /* [tokens][D] */
  const float* h0;     /* [nseq][D] or NULL */
  const float* dlast;  /* [nseq][D] or NULL */
  const void* offsets; /* [nseq + 1] or NULL */
  void* dgate;         /* [tokens][D / group] */
  void* dx;            /* [tokens][D] */
  float* dh0;          /* [nseq][D] or NULL */
  int64_t tokens;
  int64_t ld_gate, ld_x, ld_h, ld_dh, ld_dgate, ld_dx;
  int32_t nseq, D, group, dtype, offset_bytes, form, reverse;
} polyglot_recurrence_grad_args;
int polyglot_recurrence_grad(polyglot_ctx* ctx, const polyglot_recurrence_grad_args* args);

/* Sizes the recurrence's workspace for calls of up to max_tokens tokens and
 * max_D channels, of any group and storage format: about 1.2 bytes for each token and
 * channel, of max_D + 128 channels, and 11 MB (65,536 tokens of 2,048 channels: 185 MB).
 * Waits for the context's stream, frees what an earlier call
 * reserved and allocates: to be called outside of graph capture, and graphs that
 * were captured with the earlier workspace must not be replayed afterwards. */
int polyglot_reserve_recurrence(polyglot_ctx* ctx, int64_t max_tokens, int32_t max_D);

/* The scores of a vocabulary made ready for a choice, one row for each live
 * sequence, and the choice.  For every row r and word v, in this order and in
 * 32 bits:
 *
 *   l = logits[r][v]
 *   v in history[r]:            l = l > 0 ? l / repetition[r] : l * repetition[r]
 *   n times in its made part:   l = l - (frequency[r] n + presence[r])     (n > 0)
 *   l = l + bias[v]
 *   v not allowed by the mask:  l = -infinity, whatever it was
 *
 * history[r] holds the first lengths[r] ids of its row (all `history_cap` if
 * lengths is NULL); those before prompt[r] are the prompt, the others were made
 * by the model (all of them if prompt is NULL).  Negative ids are padding; ids
 * >= V raise the sticky flag (POLYGLOT_EID) and count for nothing.  Lengths and
 * prompts outside [0, history_cap] are taken as the nearer end.
 * repetition, frequency and presence are per row; NULL stands for 1, 0 and 0.
 * bias[V] is float32, shared (ld_bias 0) or one row per row.
 * A mask row is ceil(V / 32) words of 32 bits, bit v % 32 of word v / 32 set where
 * v is allowed; row r takes row mask_rows[r] (negative: no mask), or without
 * mask_rows its own (masks == rows) or the only one (masks == 1).  A mask_rows
 * entry >= masks raises the sticky flag and masks nothing.
 *
 * out receives l in dtype and may be logits (with the same ld) or NULL.
 * token[r], if not NULL, receives the word of the largest l (before its rounding
 * to dtype), the lowest one of equals; NaN is never chosen; -1 if no l is above
 * -infinity.  lse[r], if not NULL, receives log(sum_v e^l) (-infinity for a row
 * that the mask leaves empty; NaN if an l is NaN).
 * rows = 0 does nothing.  token and lse use the workspace of polyglot_reserve_logits. */
typedef struct {
  const void* logits;
  void* out;
  const int32_t* history; /* [rows][history_cap], or NULL */
  const int32_t* lengths; /* [rows] or NULL */
  const int32_t* prompt;  /* [rows] or NULL */
  const float* repetition;
  const float* presence;
  const float* frequency;
  const float* bias;
  const uint32_t* mask;
  const int32_t* mask_rows;
  int32_t* token;
  float* lse;
  int64_t ld_logits, ld_out, ld_history, ld_bias, ld_mask;
  int32_t rows;
  int32_t V;              /* 1 .. 2^30 */
  int32_t dtype, history_cap, masks;
} polyglot_logits_args;
int polyglot_logits(polyglot_ctx* ctx, const polyglot_logits_args* args);

/* Sizes the workspace that joins the parts of a row, for calls of up to max_rows
 * rows of max_V scores: 128 bytes a row, and 24 for every 1,024 of its words; otherwise as polyglot_reserve_recurrence. */
int polyglot_reserve_logits(polyglot_ctx* ctx, int32_t max_rows, int32_t max_V);

/* The operators' kernels under polyglot_set_timing, as polyglot_kernel_times
 * reports the others. */
#define POLYGLOT_OPK_DROPOUT 0
#define POLYGLOT_OPK_RECURRENCE 1
#define POLYGLOT_OPK_RECURRENCE_GRAD 2
#define POLYGLOT_OPK_LOGITS 3
#define POLYGLOT_NOPKERNELS 4
int polyglot_operator_times(polyglot_ctx* ctx, double* ms, int32_t* launches);

/* Synchronises the stream and returns the sticky device error
 * (POLYGLOT_OK, POLYGLOT_EID, POLYGLOT_EOFFSETS, or POLYGLOT_EHIP for a library
 * error or calls that overlapped), then clears it. */
int polyglot_status(polyglot_ctx* ctx);

/* Text of the last error recorded on this context ("" if none). */
const char* polyglot_last_error(const polyglot_ctx* ctx);

#ifdef __cplusplus
}
#endif

#endif /* POLYGLOT_H */
