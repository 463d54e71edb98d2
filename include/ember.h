/*
 * ember.h: C ABI of the Ember token-table optimizer step for AMD MI355X (gfx950).
 *
 * Ember (Token Geometry, Algorithm 1 in Section 2) updates a V x D
 * token-interface matrix W (embedding table or LM head) from its gradient G
 * with O(V + D) state: a row second-moment vector r (V floats) and a column
 * second-moment vector c (D floats).  One step t >= 1 computes
 *
 *   r <- beta2 r + (1 - beta2) mean_j G_ij^2          (row statistic)
 *   c <- beta2 c + (1 - beta2) mean_i G_ij^2          (column statistic)
 *   rhat = r / (1 - beta2^t),  chat = c / (1 - beta2^t)
 *   s = sqrt(mean(rhat) mean(chat))
 *   W_ij <- W_ij -/+ lr G_ij / (sqrt(rhat_i chat_j / s) + eps)
 *
 * The V x D preconditioner rhat chat^T / s is never stored: the update is
 * applied as a row scaling times a column scaling (section "Distributed
 * Ember", paragraph on the preconditioner).  All reductions use a fixed
 * order, with no floating-point atomics, so a given input produces the same
 * bits on every run (same section, on the fused deterministic reduction).
 *
 * Conventions shared by every entry point:
 *  - Memory: every pointer argument except the scalars is DEVICE memory owned
 *    by the caller.  The library never allocates, frees or synchronises,
 *    except ember_get_error (which synchronises the stream it is given).
 *  - Layout: W and G are row-major, row i starting at element i * ld.  Both
 *    base pointers must be 16-byte aligned and ld * element_size must be a
 *    multiple of 16 bytes, so every row starts on a 16-byte boundary.  Only
 *    the first D elements of each row are read or written.  W must not
 *    overlap G, r, c or the workspace.
 *  - dtypes: W and G are EMBER_F32 or EMBER_BF16, independently.  r and c are
 *    always fp32 (the paper keeps optimizer state in fp32).  Arithmetic is
 *    fp32; W is written with round-to-nearest-even; an element whose
 *    gradient is exactly zero keeps its bits.
 *  - Streams: all work is enqueued on `stream` (0 = the null stream) in
 *    order; calls return before the work runs.  One (r, c, workspace) set
 *    must not be used by two streams at once.
 *  - Errors: every argument check below happens on the host before anything
 *    is enqueued; on a negative return nothing was enqueued and no memory was
 *    touched.  EMBER_ERR_HIP means a launch failed after validation.
 *  - Step counter: t is owned by the caller: it starts at 0 and the caller
 *    passes t = 1, 2, ... (Algorithm 1 increments t before each update).
 *  - Sign: maximize = 0 descends a loss (W -= ...); maximize = 1 is the
 *    paper's literal ascent of a reward (W += ...).
 */
#ifndef EMBER_H
#define EMBER_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { EMBER_F32 = 0, EMBER_BF16 = 1 } ember_dtype;

typedef enum {
    EMBER_OK = 0,
    EMBER_ERR_ARG = -1,       /* null pointer, or a scalar out of range */
    EMBER_ERR_SHAPE = -2,     /* V or D < 1 or too large, ld < D, n_idx > V */
    EMBER_ERR_ALIGN = -3,     /* W/G not 16-byte aligned, ld*size not a multiple of 16,
                                 r/c not 4-byte aligned, workspace not 256-byte aligned */
    EMBER_ERR_DTYPE = -4,     /* dtype is not EMBER_F32 or EMBER_BF16 */
    EMBER_ERR_WORKSPACE = -5, /* ws_bytes smaller than ember_workspace_bytes(V, D) */
    EMBER_ERR_INDEX = -6,     /* sparse step: idx holds a value outside [0, V) or a
                                 repeated value, or a device row count is out of
                                 range (reported by ember_get_error) */
    EMBER_ERR_HIP = -7,       /* a HIP runtime call failed */
    EMBER_ERR_DEVICE = -8     /* sparse step (reported by ember_get_error): the blocks of
                                 the one-launch form did not all run at once, so a grid
                                 barrier's bounded wait ran out; W, r and c are then
                                 unspecified.  Not expected on an MI355X that the
                                 calling process has to itself. */
} ember_status;

/* Largest supported V (row indices are kept in 31 bits) and D, and the
 * largest token batch of ember_coalesce_rows. */
#define EMBER_MAX_V ((int64_t)0x7FFFFFFE)
#define EMBER_MAX_D ((int64_t)(1 << 22))
#define EMBER_MAX_TOKENS ((int64_t)(1 << 26))
/* ember_lmhead_step: row strides of dY and H below 2^24 elements (the slice of
 * one token step of either is then addressable with 32-bit offsets), and at
 * most 2^30 tokens. */
#define EMBER_LMHEAD_MAX_LD ((int64_t)(1 << 24))
#define EMBER_LMHEAD_MAX_T ((int64_t)(1 << 30))

/*
 * Workspace size for a V x D table, valid for every step (dense, sparse,
 * canonical and row-only).  The workspace holds the per-block partial sums of the fixed-order
 * reductions, a V-entry row-slot table used by the sparse step, and a status
 * word.  It is caller-allocated device memory, 256-byte aligned, and must be
 * initialised once by ember_init_state before its first step.
 * Returns EMBER_OK and sets *bytes, or EMBER_ERR_SHAPE / EMBER_ERR_ARG.
 */
int ember_workspace_bytes(int64_t V, int64_t D, size_t* bytes);

/*
 * Ember state initialisation (Algorithm 1: r_0 = 0 in R^V, c_0 = 0 in R^D,
 * t = 0).  Enqueues zero fills of r (V floats), c (D floats) and the parts
 * of the workspace that must start at zero.  The caller sets t = 0.
 */
int ember_init_state(float* r, float* c, int64_t V, int64_t D,
                     void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * One dense Ember step (Algorithm 1, one pass of its loop body) on W (V x D,
 * row stride ldw, dtype w_dtype) with gradient G (V x D, row stride ldg,
 * dtype g_dtype).  r (V) and c (D) are updated in place, then W.
 * Scalars: t >= 1; lr >= 0 and finite; 0 <= beta2 < 1; eps >= 0 and finite
 * (the paper's defaults: lr = 1e-3, beta2 = 0.999, eps = 1e-8).  beta2 is
 * used as the fp32 value passed.
 */
int ember_step_dense(void* W, int w_dtype, int64_t ldw,
                     const void* G, int g_dtype, int64_t ldg,
                     float* r, float* c, int64_t V, int64_t D, int64_t t,
                     float lr, float beta2, float eps, int maximize,
                     void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * One sparse-row Ember step: the gradient is zero except on the n_idx rows
 * listed in idx (the embedding-table case of Section 2.2, where only the
 * tokens of the batch receive gradient).  G_rows is n_idx x D (row stride
 * ldg, compact: row k is the gradient of W's row idx[k]).  idx is a device
 * array of n_idx int64 values, unique and in [0, V), in any order;
 * n_idx = 0 is allowed (then G_rows and idx may be NULL).
 *
 * The result is the dense step on the gradient that is zero outside idx:
 * every row's r decays by beta2 (touched rows also add their statistic), the
 * column mean still divides by V, s uses all V rows, and W rows outside idx
 * are not touched.
 *
 * Index errors (a value outside [0, V), or a repeated value) are detected on
 * the device: the step then leaves W, r and c unchanged, and the next
 * ember_get_error on this workspace reports EMBER_ERR_INDEX.  The caller
 * should then not advance t.
 */
int ember_step_sparse_rows(void* W, int w_dtype, int64_t ldw,
                           const void* G_rows, int g_dtype, int64_t ldg,
                           const int64_t* idx, int64_t n_idx,
                           float* r, float* c, int64_t V, int64_t D, int64_t t,
                           float lr, float beta2, float eps, int maximize,
                           void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * The sparse step with its row count in device memory, for callers whose
 * count is produced on the device (ember_coalesce_rows writes it): nothing is
 * read back to the host, so coalescing and the step can be enqueued together
 * or captured in one HIP graph.  n_idx_dev points to one int64 in device
 * memory, read when the step runs; max_rows (host) bounds it and sizes the
 * launches; G_rows and idx must hold max_rows rows.  A device count outside
 * [0, max_rows] is reported like an index error (EMBER_ERR_INDEX through
 * ember_get_error; W, r and c untouched).  The step takes the one-launch form
 * of ember_step_sparse_rows whenever the count fits it: decided on the host
 * when max_rows fits, else on the device from the count (the one-launch kernel
 * runs first and, when it has taken the step, the three launches of the other
 * form return at once).  With *n_idx_dev == max_rows, or a count that takes the
 * one-launch form, the result is the same, bit for bit, as
 * ember_step_sparse_rows with n_idx = that count; other counts partition the
 * rows differently and agree within the stated tolerances.  Everything else as
 * for ember_step_sparse_rows.
 */
int ember_step_sparse_rows_devn(void* W, int w_dtype, int64_t ldw,
                                const void* G_rows, int g_dtype, int64_t ldg,
                                const int64_t* idx, const int64_t* n_idx_dev, int64_t max_rows,
                                float* r, float* c, int64_t V, int64_t D, int64_t t,
                                float lr, float beta2, float eps, int maximize,
                                void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * The sparse-row step without a workspace argument, for callers that cannot
 * allocate device memory: code under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation.  The step is ember_step_sparse_rows's
 * one-launch form (same kernel, same bits as that call with a workspace); its
 * scratch (row marks, barrier flags, per-block partial sums, column factors)
 * is a 16 MiB array inside the library, one per GPU, held until the process
 * ends.  Each call enqueues a small zero fill of that array's first part and
 * of *status, then the step; nothing is allocated.
 *
 * Arguments as for ember_step_sparse_rows (W, G_rows, idx, n_idx, r, c, V, D,
 * t and the scalars), without ws/ws_bytes, plus:
 *   status  device int32 (4-byte aligned, required): set to 0 by the call's
 *           fill, then the step ORs its error bits into it (1: an id outside
 *           [0, V), 2: a repeated id; W, r and c are then unchanged; 8: the
 *           step's blocks did not all run at once, W, r and c unspecified).
 *           Read it after the stream has reached the step.
 * r and c start at zero (Algorithm 1's r_0, c_0) and are the caller's, as is t.
 *
 * Limits (checked on the host before anything is enqueued):
 *   the step's scratch, about 4 V + 1028 D bytes + 23 KiB, at most 16 MiB
 *   (e.g. V up to 3.1 million rows at D = 4096): EMBER_ERR_WORKSPACE otherwise;
 *   the one-launch form must take the step: D a whole number of 16-byte chunks
 *   of G, at most 8 column slabs of 2 KiB (bf16 D <= 8192, fp32 D <= 4096),
 *   n_idx within the rows held on chip (5120 at 4096 bf16 columns), and a
 *   device that keeps 256 blocks of the kernel resident: EMBER_ERR_SHAPE
 *   otherwise.
 * Calls that overlap on one GPU (two streams, or two threads) share the array
 * and race; calls must be ordered.
 */
int ember_step_sparse_rows_static(void* W, int w_dtype, int64_t ldw,
                                  const void* G_rows, int g_dtype, int64_t ldg,
                                  const int64_t* idx, int64_t n_idx,
                                  float* r, float* c, int64_t V, int64_t D, int64_t t,
                                  float lr, float beta2, float eps, int maximize,
                                  int32_t* status, hipStream_t stream);

/*
 * Several Ember steps in one call: the tables of a model (for example the
 * LM head, dense, and the input embedding, sparse rows) each take the step
 * Algorithm 1 defines for them (or the row-only step of Section 2.1), exactly
 * as the single-table entry points would, but the canonical tables share
 * three launches (one statistics pass, one finalize pass, one apply pass over
 * every table) instead of three per table, so the tables share the chip and a
 * small table costs its bytes instead of its launch latency; a sparse table
 * whose rows fit on chip takes its one-launch step (that of
 * ember_step_sparse_rows) ahead of them.  Each table's results are the same bits as its own
 * single-table call (ember_step_dense, ember_step_sparse_rows(_devn), or the
 * row-only entry points declared below).
 *
 * One ember_table_step per table:
 *   W, w_dtype, ldw, G, g_dtype, ldg, r, c, V, D, t, lr, beta2, eps,
 *   maximize, ws, ws_bytes   as for ember_step_dense;
 *   sparse = 0               dense step: G is V x D; idx, n_idx, n_idx_dev unused;
 *   sparse = 1               sparse-row step: G holds n_idx compact rows of the
 *                            rows idx lists, as for ember_step_sparse_rows;
 *                            with n_idx_dev non-NULL the row count is read from
 *                            that device int64 when the step runs and n_idx is
 *                            its maximum, as for ember_step_sparse_rows_devn.
 *   row_only = 1             the row-only step of that table (state r only; c
 *                            may be NULL), as ember_rowonly_step_dense /
 *                            ember_rowonly_step_sparse_rows(_devn) would take
 *                            it: the sparse row-only tables' id checks share one
 *                            launch and the row-only passes one more.
 * Tables may differ in every field (shape, dtypes, scalars, t).  Tables with
 * the same dtypes and the same columns-per-lane plan share launches; others
 * add launches of their own.
 *
 * Errors: each table is checked as its own call would be, and additionally
 * no memory one table writes (workspace, r, c, W) may overlap memory another
 * table reads or writes (those, and G, idx, the device row count), since the
 * tables share launches (EMBER_ERR_ARG); memory the tables only read may be
 * shared.  1 <= n_tables <= EMBER_MAX_TABLES (EMBER_ERR_ARG).  A failed check enqueues nothing for any table.  Index
 * errors of a sparse table leave that table untouched (the others step
 * normally) and are reported by ember_get_error on its workspace.
 */
#define EMBER_MAX_TABLES 8

typedef struct {
    void* W;
    int w_dtype;
    int64_t ldw;
    const void* G;
    int g_dtype;
    int64_t ldg;
    int sparse;
    int row_only;
    const int64_t* idx;
    int64_t n_idx;
    const int64_t* n_idx_dev;
    float* r;
    float* c;
    int64_t V;
    int64_t D;
    int64_t t;
    float lr;
    float beta2;
    float eps;
    int maximize;
    void* ws;
    size_t ws_bytes;
} ember_table_step;

int ember_step_multi(const ember_table_step* tables, int n_tables, hipStream_t stream);

/*
 * Row-only Ember (Section 2.1, the variant the paper analyses most, listed in
 * its ablation table with V floats of state): only the row statistic r is
 * kept, and each row's gradient is divided by the square root of its own
 * bias-corrected statistic:
 *
 *   r <- beta2 r + (1 - beta2) mean_j G_ij^2,   rhat = r / (1 - beta2^t)
 *   W_ij <- W_ij -/+ lr G_ij / (sqrt(rhat_i) + eps)
 *
 * (the canonical step with vtil_ij = rhat_i: no column statistic and no
 * normaliser s).  Each row is then independent of the others, so the step is
 * one pass that reads G and W once and writes W once.  Arguments, layouts,
 * dtypes, streams and error handling are those of the canonical entry points
 * above, without c.  The workspace is sized by ember_workspace_bytes(V, D)
 * and may be shared with nothing else while in use.
 */

/* Row-only state initialisation: zero fills of r (V floats) and of the parts
 * of the workspace that must start at zero.  The caller sets t = 0. */
int ember_rowonly_init_state(float* r, int64_t V, int64_t D,
                             void* ws, size_t ws_bytes, hipStream_t stream);

/* One dense row-only step on W (V x D) with gradient G (V x D); r is updated
 * in place, then W.  Scalar ranges as for ember_step_dense. */
int ember_rowonly_step_dense(void* W, int w_dtype, int64_t ldw,
                             const void* G, int g_dtype, int64_t ldg,
                             float* r, int64_t V, int64_t D, int64_t t,
                             float lr, float beta2, float eps, int maximize,
                             void* ws, size_t ws_bytes, hipStream_t stream);

/* One sparse-row row-only step (G_rows, idx and n_idx as for
 * ember_step_sparse_rows): the dense row-only step on the gradient that is zero
 * outside idx.  Rows outside idx only see r decay by beta2; their W rows are
 * not touched.  Index errors leave W and r unchanged and are reported by
 * ember_get_error. */
int ember_rowonly_step_sparse_rows(void* W, int w_dtype, int64_t ldw,
                                   const void* G_rows, int g_dtype, int64_t ldg,
                                   const int64_t* idx, int64_t n_idx,
                                   float* r, int64_t V, int64_t D, int64_t t,
                                   float lr, float beta2, float eps, int maximize,
                                   void* ws, size_t ws_bytes, hipStream_t stream);

/* The row-only sparse step with its row count in device memory (as for
 * ember_step_sparse_rows_devn). */
int ember_rowonly_step_sparse_rows_devn(void* W, int w_dtype, int64_t ldw,
                                        const void* G_rows, int g_dtype, int64_t ldg,
                                        const int64_t* idx, const int64_t* n_idx_dev, int64_t max_rows,
                                        float* r, int64_t V, int64_t D, int64_t t,
                                        float lr, float beta2, float eps, int maximize,
                                        void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * Gradient coalescing: the step before ember_step_sparse_rows.  The gradient
 * of an input embedding for one batch position is the one-hot selector of its
 * token times the back-propagated signal (appendix "Decomposing the Squared
 * Gradient"), so the gradient of row i is the sum of the signals of every
 * position holding token i (appendix "The Fisher is Proportional to Inverse
 * Frequency Squared").  Given n_tok token ids tok (device int64, each in
 * [0, V)) and the per-position signals U (n_tok x D, row stride ldu, dtype
 * u_dtype), this writes
 *
 *   *n_out           n, the number of distinct ids (device int64);
 *   idx[0..n)        the distinct ids, ascending (device int64[n_tok]);
 *   G_rows[k][0..D)  for k < n: the sum of U[p] over the positions p with
 *                    tok[p] == idx[k], accumulated in float64 and rounded once
 *                    (nearest-even) to g_dtype (device, n_tok x D, stride ldg).
 *
 * The sums have a fixed order, so results are reproducible bit for bit: the
 * positions of one id are added in ascending order, within fixed chunks of the
 * id-sorted positions, and chunk partials in chunk order.  idx and G_rows feed
 * ember_step_sparse_rows directly once n is known on the host (read *n_out
 * after synchronising the stream), or feed ember_step_sparse_rows_devn with
 * n_out itself.  Ids outside [0, V) make the call report EMBER_ERR_INDEX
 * through ember_get_error on this workspace and write n = -1 (which a
 * device-count step refuses, leaving its table untouched); idx and G_rows are
 * then unspecified.  n_tok = 0 gives n = 0 (tok, U, idx, G_rows may
 * then be NULL).  Layout and alignment rules of U and G_rows are those of W
 * and G; tok, idx and n_out must be 8-byte aligned.
 *
 * The workspace (device, 256-byte aligned, ember_coalesce_workspace_bytes of
 * at least n_tok tokens) needs no initialisation and may be reused by
 * successive calls on one stream; its size grows with max_tokens (sort
 * buffers) and with D (float64 partial rows of at most 2^25 elements).
 */
int ember_coalesce_workspace_bytes(int64_t max_tokens, int64_t V, int64_t D, size_t* bytes);

int ember_coalesce_rows(const int64_t* tok, int64_t n_tok,
                        const void* U, int u_dtype, int64_t ldu,
                        int64_t V, int64_t D,
                        int64_t* idx, void* G_rows, int g_dtype, int64_t ldg,
                        int64_t* n_out, void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * LM-head step with the gradient statistics taken inside the weight-gradient
 * GEMM.  For an LM head with logits z_m = W h_m, the cross-entropy gradient of
 * row i is G_i = sum_m (q_mi - 1[y_m = i]) h_m (appendix "The LM Head
 * Factorizes Like the Embedding Table"): G = dY^T H, with dY (T x V, row
 * stride ldy) the gradient of the logits and H (T x D, row stride ldh) the
 * hidden states, both bf16, token-major as a forward pass produces them.
 *
 * The call computes G with bf16 matrix instructions and fp32 accumulation,
 * rounds it once (nearest-even) to g_dtype and stores it in G (V x D, row
 * stride ldg; the caller keeps it, e.g. for clipping or logging), and takes
 * the dense Ember step on W with that G.  The result is that of
 * ember_step_dense(W, G, ...) on the stored G, up to the summation order of
 * the row and column sums of g^2, which here are formed by the GEMM's
 * epilogue from the stored values (fixed order, bit-reproducible), so the
 * step does not read G a second time for its statistics.
 *
 * T = 0 is allowed (G = 0; dY and H may then be NULL).  W, G, r, c, t, the
 * scalars, the workspace (ember_workspace_bytes(V, D), initialised by
 * ember_init_state) and the error rules are those of ember_step_dense;
 * additionally dY and H follow the layout rules of W and G, ldy and ldh must
 * be below EMBER_LMHEAD_MAX_LD and T at most EMBER_LMHEAD_MAX_T
 * (EMBER_ERR_SHAPE otherwise).  G must not overlap dY, H, W or the state.
 * The row-stride padding of dY and H (columns V..ldy-1 and D..ldh-1) is read
 * but never affects a stored value.
 */
int ember_lmhead_step(void* W, int w_dtype, int64_t ldw,
                      const void* dY, int64_t ldy, const void* H, int64_t ldh, int64_t T,
                      void* G, int g_dtype, int64_t ldg,
                      float* r, float* c, int64_t V, int64_t D, int64_t t,
                      float lr, float beta2, float eps, int maximize,
                      void* ws, size_t ws_bytes, hipStream_t stream);

/* Row strides of 8-bit codes below 2^22 bytes (the rows of one tile are then
 * addressable with 32-bit offsets). */
#define EMBER_Q8_MAX_LD ((int64_t)(1 << 22))

/*
 * The final norm: a residual addition, a root-mean-square norm and, where the
 * rows go to an 8-bit head, their rounding to 8 bits, in one pass.  For each of
 * T rows of D columns
 *
 *   s = x + r                                  (r: the residual stream; may be NULL)
 *   rstd = 1 / sqrt(mean_j s_j^2 + eps)
 *   y_j = s_j rstd gain_j
 *   a = max_j |y_j|,  qscale = a / 127,  q_j = rint(y_j 127 / a)
 *
 * Arithmetic is fp32 and y is formed from the unrounded sum.  Outputs, each
 * NULL if it is not wanted, at least one of Y and Q:
 *   S (T x D, x_dtype)   the sum, with R only; it may be X or R itself (same ld);
 *   Y (T x D, y_dtype)   the norm's output (the H of ember_lmhead_step); it may
 *                        be X itself (same dtype and ld) where S is not;
 *   Q (T x D, int8) and qscale (T), both or neither: y in 8 bits, codes in
 *                        [-127, 127], one scale a row.  A row whose a is below
 *                        1e-36 (zeros among them) has codes and scale 0; one
 *                        that holds an infinity or a NaN has codes 0 and scale
 *                        NaN, which makes its logits NaN;
 *   rstd (T)             kept for the gradient.
 * The mean square of a finite row is right over the whole range of x_dtype, also where
 * squares leave that of fp32.  With an eps that does not bound it, rstd itself is infinite
 * for rows whose root mean square is below 3e-39 (y is then not finite).
 * X, R (x_dtype), S, Y: layout rules of W and G; between two rows the padding up to
 * the next 16-byte boundary may be read, its values do not matter.  Q: 16-byte aligned, ldq a
 * multiple of 16 below EMBER_Q8_MAX_LD; columns D..ldq-1 are not written.  gain: D values of
 * gain_dtype, 16-byte aligned.  An output shares no memory with another argument other
 * than as said (EMBER_ERR_ARG; columns of one buffer at one stride are fine).
 * 0 <= T <= EMBER_MAX_TOKENS (0: nothing to do, the pointers may be NULL), 1 <= D <= EMBER_NORM_MAX_D, eps >= 0 and finite.
 */
#define EMBER_NORM_MAX_D ((int64_t)32768)

int ember_rmsnorm(const void* X, int x_dtype, int64_t ldx, const void* R, int64_t ldr,
                  const void* gain, int gain_dtype, float eps, int64_t T, int64_t D,
                  void* S, int64_t lds, void* Y, int y_dtype, int64_t ldy,
                  int8_t* Q, int64_t ldq, float* qscale, float* rstd, hipStream_t stream);

/*
 * The norm's gradient.  S (T x D, x_dtype) is the sum the forward call stored
 * (or its X, without R) and rstd what it wrote; dY (T x D, x_dtype) the gradient
 * of Y; dS (T x D, x_dtype, may be NULL) a gradient that reaches the sum by
 * another way, such as the residual stream.  With u = dy gain and h = s rstd:
 *
 *   dx_j = rstd (u_j - mean_k(u_k h_k) h_j) + ds_j    -> dX (T x D, x_dtype)
 *   dgain_j = sum_t dy_tj h_tj                        -> dgain (D, fp32)
 *
 * dX is the gradient of X and of R; it may be dY, dS or S itself (same ld) and
 * shares no other memory with an argument.  dgain is overwritten (zeros for T = 0);
 * its sum has an order fixed by T, D and x_dtype.  The workspace (device, 256-byte
 * aligned, ember_rmsnorm_grad_workspace_bytes of at least T tokens and this D) needs
 * no initialisation.
 */
int ember_rmsnorm_grad_workspace_bytes(int64_t max_tokens, int64_t D, size_t* bytes);

int ember_rmsnorm_grad(const void* dY, int64_t lddy, const void* S, int x_dtype, int64_t lds,
                       const void* gain, int gain_dtype, const float* rstd, const void* dS, int64_t ldds,
                       int64_t T, int64_t D, void* dX, int64_t lddx, float* dgain,
                       void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * Rows of a table in 8 bits, as the norm writes Q and qscale, from the rows
 * themselves: what ember_logits_q8 reads as Wq and wscale.  1 <= D <=
 * EMBER_NORM_MAX_D, 0 <= rows <= EMBER_MAX_V (0: nothing to do, the pointers may
 * be NULL).
 */
int ember_quantize_rows(const void* X, int x_dtype, int64_t ldx, int64_t rows, int64_t D,
                        int8_t* Q, int64_t ldq, float* qscale, hipStream_t stream);

/*
 * Logits of an LM head held in 8 bits, for T tokens:
 *
 *   Y_tv = (sum_k Xq_tk Wq_vk) xscale_t wscale_v + bias_v
 *
 * Xq (T x D) and Wq (V x D) are int8 codes with one fp32 scale a row (xscale: T,
 * wscale: V), bias (V, fp32) may be NULL, Y is T x V of y_dtype.  The sum over D
 * is exact (int32), the scaling fp32, and the result is rounded once to y_dtype.
 * Layout: bases 16-byte aligned, ldx and ldw multiples of 16 below
 * EMBER_Q8_MAX_LD, Y as W and G.  The padding of Xq and Wq (columns D..ld-1) may
 * be read but never affects a stored value.  0 <= T <= EMBER_MAX_TOKENS (0:
 * nothing to do, the pointers may be NULL), 1 <= V <= EMBER_MAX_V, 1 <= D <=
 * EMBER_NORM_MAX_D.
 */
int ember_logits_q8(const int8_t* Xq, int64_t ldx, const float* xscale,
                    const int8_t* Wq, int64_t ldw, const float* wscale, const float* bias,
                    int64_t T, int64_t V, int64_t D, void* Y, int y_dtype, int64_t ldy, hipStream_t stream);

/*
 * Tables in 4 bits, for answering: the head and the embedding of a model whose
 * every token reads them.  A row's columns are in groups of 32, 64 or 128 (the
 * last one may be shorter), each with a bf16 scale:
 *
 *   a = max |x| of the group,  s = bf16(a (1/7)),  c = rint(x / s) in [-7, 7]
 *
 * in fp32: the product with the fp32 nearest 1/7 is rounded to fp32, then to bf16, the
 * quotient correctly rounded to fp32, then to the nearest integer, to even at a tie.
 * A group whose a is below 1e-36 (zeros among them) has codes and scale 0; one that
 * holds an infinity or a NaN has codes 0 and scale NaN.  Codes are in two's
 * complement, so a table made elsewhere may hold -8 too, and any scales.
 *
 * Packing (Wq, Q): the 128 columns from 128 i on take the 64 bytes from 64 i on of
 * their row.  Byte 16 q + 4 w + b of them (q, w, b in 0..3) holds the code of column
 * 128 i + 32 w + 4 q + b in its lower half and that of the column 16 further in its
 * upper half.  A row takes 64 ceil(D / 128) bytes; ember_quantize_rows_q4 writes all of
 * them (codes 0 past column D), ember_rows_q4 and ember_logits_q4 may read the codes
 * past column D, but these never affect a stored value, nor does padding.
 * Layout: codes 16-byte aligned, their row stride in bytes a multiple of 16 below
 * EMBER_Q8_MAX_LD; scales (bf16 bits, one row of ceil(D / group) for each of the
 * table's) 16-byte aligned, their row stride a multiple of 8 below EMBER_Q8_MAX_LD.
 * X, Y: layout rules of W and G.  1 <= V (rows) <= EMBER_MAX_V, 1 <= D <=
 * EMBER_NORM_MAX_D; outputs share no memory with another argument (EMBER_ERR_ARG), and a
 * group of another size is EMBER_ERR_ARG too.
 *
 * ember_quantize_rows_q4: rows of X in 4 bits.  rows = 0: nothing to do, the pointers
 * may be NULL.
 */
int ember_quantize_rows_q4(const void* X, int x_dtype, int64_t ldx, int64_t rows, int64_t D, int group,
                           uint8_t* Q, int64_t ldq, uint16_t* gscale, int64_t lds, hipStream_t stream);

/*
 * Rows read back from 4 bits: Y_i = the values of row tok_i (device int64[n]), or of
 * row i with tok NULL (then n <= V).  A value is the product of a code and its scale,
 * rounded once to y_dtype.  A token outside [0, V) gives a row of NaN.  0 <= n <=
 * EMBER_MAX_TOKENS with tok (0: nothing to do, the pointers may be NULL).
 */
int ember_rows_q4(const uint8_t* Wq, int64_t ldw, const uint16_t* wscale, int64_t lds, int group,
                  int64_t V, int64_t D, const int64_t* tok, int64_t n,
                  void* Y, int y_dtype, int64_t ldy, hipStream_t stream);

/*
 * Logits of an LM head held in 4 bits, for T tokens in 8 (Xq and xscale as
 * ember_logits_q8 has them):
 *
 *   Y_tv = xscale_t sum_g wscale_vg (sum_{k in g} Xq_tk c_vk) + bias_v
 *
 * A group's sum is exact, the sum over the groups fp32 in an order fixed by the sizes
 * (held times 16: one of 2^124 and more is an infinity); the result is rounded once to
 * y_dtype.  bias (V, fp32) may be NULL.  0 <= T <= EMBER_MAX_TOKENS (0: nothing to do,
 * the pointers may be NULL).
 */
int ember_logits_q4(const int8_t* Xq, int64_t ldx, const float* xscale,
                    const uint8_t* Wq, int64_t ldw, const uint16_t* wscale, int64_t lds, int group,
                    const float* bias, int64_t T, int64_t V, int64_t D,
                    void* Y, int y_dtype, int64_t ldy, hipStream_t stream);

/*
 * A token drawn from each of T rows of V logits (L, T x V, of l_dtype; minus infinity:
 * a token that is not allowed).  Row t has a temperature, top-k, top-p, min-p (arrays
 * of T on the device, each NULL if no row has it) and a random number u_t.  With
 * e_i = exp((l_i - max l) / temperature):
 *
 *   top-k   keeps the k first tokens in falling order of l (equal ones by index); 0: all
 *   top-p   of those, the shortest prefix whose e sum to p times their sum at least (the
 *           first token always); 1: all
 *   min-p   of those, the tokens with e_i >= min_p; 0: all
 *   id      the first token, by index, at which the running sum of the kept e is above
 *           u times their sum
 *
 * Temperature 0 takes the first of the largest logits (temperature 1 and k = 1).
 * Outputs: ids (T, int64); logp (T, may be NULL): the log of e_id over the sum of all
 * e, that is before the filters; kept (T, may be NULL): the number of tokens kept.  A
 * row that has nothing to draw from (no logit above minus infinity), that holds a NaN
 * or an infinity, or whose parameters are out of range (temperature >= 0 and finite,
 * k >= 0, 0 <= p <= 1, 0 <= min_p <= 1, 0 <= u < 1) has id -1, logp NaN and kept 0.
 * e are held in fixed point, to less than 2^-n with n = min(48, 62 - ceil(log2 V)):
 * a token whose e is below half of that is never drawn.  The result depends on a row's logits
 * and parameters alone, and has the same bits on every run.
 * Layout: L as W and G; 0 <= T <= EMBER_MAX_TOKENS (0: nothing to do, the pointers may
 * be NULL), 1 <= V <= EMBER_SAMPLE_MAX_V.  Outputs and the workspace share no memory
 * with another argument (EMBER_ERR_ARG).  The workspace (device, 256-byte aligned,
 * ember_sample_workspace_bytes of at least T tokens and this V) needs no
 * initialisation; calls that share one must not run at once.  Rows of up to 8192
 * tokens leave it as it is, and 4 KiB serve any number of them.
 */
#define EMBER_SAMPLE_MAX_V ((int64_t)1 << 24)

int ember_sample_workspace_bytes(int64_t max_tokens, int64_t V, size_t* bytes);

int ember_sample(const void* L, int l_dtype, int64_t ldl, int64_t T, int64_t V, const float* temperature,
                 const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                 int64_t* ids, float* logp, int32_t* kept,
                 void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * Global gradient norm and clipping.  Over all n_grads tensors together
 *
 *   norm = sqrt(sum g^2),   factor = max_norm / norm if norm > max_norm, else 1
 *   dst = factor src        (rounded once to dst_dtype)
 *
 * and out[0] = norm, out[1] = factor (device, fp32), with no host read: the
 * tables' steps can follow on the stream at once.  A norm that is NaN or
 * infinite gives factor 1.  Squares are summed in float64 in a fixed order; of
 * finite gradients the sum is finite, and so the factor below 1, also where out[0], an
 * fp32 number, reads infinity.
 *
 * One ember_grad per tensor: rows x cols elements, row i at element i * ld;
 *   src, src_dtype, lds   the gradient, aligned to its element size (views at
 *                         any element of a bucket are fine);
 *   dst, dst_dtype, ldd   where it goes: src itself (same dtype and ld; then its
 *                         rows are left alone when factor is 1) or other memory,
 *                         of either dtype;
 *   rows_dev              NULL, or a device int64 (8-byte aligned) that says how
 *                         many of the rows hold a gradient (ember_coalesce_rows
 *                         writes it); the others are not read, and zeros are
 *                         written in their place in dst.  A value outside
 *                         [0, rows] counts as the nearer end.
 * Tensors must not overlap each other's memory (not checked), nor out, the workspace
 * or a row count (EMBER_ERR_ARG).  rows, cols >= 0 (an empty
 * tensor's pointers may be NULL), rows * cols <= 2^40, 0 <= n_grads <=
 * EMBER_MAX_GRADS, max_norm >= 0 (infinite: only the norm, and copies).  The
 * workspace (device, 256-byte aligned, ember_clip_workspace_bytes(n_grads))
 * needs no initialisation.  grads is read before the call returns.
 */
#define EMBER_MAX_GRADS ((int64_t)(1 << 16))

typedef struct {
    const void* src;
    int src_dtype;
    int64_t lds;
    void* dst;
    int dst_dtype;
    int64_t ldd;
    int64_t rows;
    int64_t cols;
    const int64_t* rows_dev;
} ember_grad;

int ember_clip_workspace_bytes(int64_t n_grads, size_t* bytes);

int ember_clip_grads(const ember_grad* grads, int64_t n_grads, float max_norm, float* out,
                     void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * Device status of the most recent step enqueued with this workspace.
 * Synchronises `stream`, then sets *device_status to EMBER_OK or
 * EMBER_ERR_INDEX.  Returns EMBER_OK, EMBER_ERR_ARG or EMBER_ERR_HIP.
 */
int ember_get_error(const void* ws, hipStream_t stream, int* device_status);

/* Static description of a status code (never NULL). */
const char* ember_strerror(int status);

/*
 * Kernel timing (diagnostics).  While enabled, each kernel the library
 * launches is bracketed by two HIP events recorded on its stream.
 * ember_profile_collect waits for those events, writes per-kernel totals
 * (name, launch count, summed duration in milliseconds) for up to
 * max_entries kernels, sets *n_entries, and clears the record.
 */
typedef struct {
    const char* name;
    int64_t launches;
    double total_ms;
} ember_kernel_stat;

int ember_profile_enable(int enable);

/*
 * Bound of each grid-barrier wait of the one-launch sparse step
 * (diagnostics, for testing its failure path): `ticks` of the GPU's 100 MHz
 * real-time counter, for the steps enqueued after the call, process-wide;
 * 0 restores the default (1e8 ticks, about one second).  A wait that runs
 * out ends the launch normally and sets the timeout bit that
 * ember_get_error reports as EMBER_ERR_DEVICE (the state is then unspecified
 * until ember_init_state).  Returns EMBER_ERR_ARG for ticks < 0, else
 * EMBER_OK.
 */
int ember_set_barrier_wait_ticks(int64_t ticks);

/*
 * Streaming probe (diagnostics): reference rates of plain streaming kernels
 * over the same bytes as the passes above (not ceilings: the passes keep more
 * rows in flight per wavefront, and the apply pass finds part of G in the
 * last-level cache, so it runs faster than mode 2).  Enqueues one grid-stride
 * kernel with 16-byte non-temporal accesses over `bytes` bytes of each operand:
 *   mode 0: reads a (dst receives at most 4 bytes, in practice none);
 *   mode 1: dst <- a (copy);
 *   mode 2: dst <- a + b in 32-bit integer lanes (two reads, one write, as
 *           the apply pass reads G and W and writes W).
 * dst, a (and b for mode 2) are device pointers, 16-byte aligned, each
 * covering `bytes`, which must be a multiple of 16; dst must not overlap a
 * or b.  Returns EMBER_ERR_ARG (mode or null pointer), EMBER_ERR_SHAPE,
 * EMBER_ERR_ALIGN, EMBER_ERR_HIP or EMBER_OK.
 */
int ember_stream_probe(int mode, void* dst, const void* a, const void* b, size_t bytes, hipStream_t stream);
int ember_profile_collect(ember_kernel_stat* out, int max_entries, int* n_entries);

#ifdef __cplusplus
}
#endif

#endif /* EMBER_H */
