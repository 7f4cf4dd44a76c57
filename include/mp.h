/* mp.h -- C ABI of the mixed-precision training step of a stack of linear layers,
 * for NVIDIA B200 (sm_100a) only.
 *
 * The operations are those of the paper "Mixed-Precision Training for NLP and Speech
 * Recognition with OpenSeq2Seq" (arXiv 1805.10387), Section 3:
 *   Section 3.1  matrix products with FP16 operands and FP32 accumulation; a loss scale S
 *                chosen from an inspection of the gradients and applied to the next step;
 *                an FP32 master copy of the weights;
 *   Section 3.2  FP16 gradients converted to FP32, optimizer run on the FP32 master,
 *                master converted back to the FP16 working copy;
 *   Section 3.3  weight decay formed from the FP32 master, not from the FP16 copy.
 *
 * Conventions
 *   - Every matrix is row-major.  FP16 means IEEE binary16 stored as 16-bit words.
 *   - Every tensor pointer is a DEVICE pointer owned by the caller and must be 16-byte
 *     aligned; leading dimensions (ld*) are in elements and multiples of 8.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  All work is
 *     asynchronous on that stream; only mp_state_read* synchronise.
 *   - Every function returns an mp_status.  Nothing throws or aborts.  Argument errors are
 *     found on the host before anything is launched.  Numeric overflow is NOT an error: it
 *     is state (found_inf, skipped) held on the device.
 *   - FP32 -> FP16 conversions round to nearest even, overflow to +-inf (never saturate)
 *     and keep subnormals.
 *   - The library owns only mp_state and mp_update_plan objects.  It runs on the device
 *     that is current when a function is called; objects belong to the device they were
 *     created on.
 *   - Calls may come from several host threads.  The one-time set-up that a first call does per
 *     device and per kernel flavour (attribute, occupancy and symbol queries) is serialised
 *     inside the library; a state or plan object must not be used by two threads at once.
 *   - Device-side errors.  Every wait inside a kernel is bounded.  A product kernel whose wait
 *     runs out stops taking work, releases what it holds and returns; it records
 *     MP_ERR_TIMEOUT in a device-wide status word and, when the call was given a state, in
 *     state->status.  While either is set, mp_master_update writes nothing and
 *     mp_loss_scale_update changes nothing (it copies the device-wide word into
 *     state->status): the training state is frozen as it was before the faulty step.  The host
 *     learns of it from mp_state_read (status) or mp_gemm_device_status, and resumes with
 *     mp_gemm_device_status (which clears the device-wide word) followed by mp_state_write
 *     with status = 0.
 *   - Token ids live in device memory, so only a kernel can see that one is out of range.  It
 *     reads nothing through such an id, marks the row's outputs (see the calls) and records
 *     MP_ERR_INVALID_ARG in state->status when the call was given a state, which freezes the
 *     training state as above.
 */
#ifndef MP_H_
#define MP_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MP_OK = 0,
  MP_ERR_INVALID_ARG = -1,      /* null pointer, non-positive size, ld < extent, bad enum  */
  MP_ERR_ALIGNMENT = -2,        /* pointer not 16-byte aligned or ld not a multiple of 8   */
  MP_ERR_UNSUPPORTED_ARCH = -3, /* current device is not compute capability 10.x           */
  MP_ERR_CUDA = -4,             /* a CUDA runtime/driver call failed; see mp_last_error    */
  MP_ERR_TIMEOUT = -5,          /* a bounded device-side wait expired (reported in status) */
  MP_ERR_NOMEM = -6,            /* allocation failed or workspace too small                */
  MP_ERR_TOO_LARGE = -7         /* size beyond a stated maximum                            */
} mp_status;

typedef struct mp_state mp_state;             /* device-resident scaler + flag + log        */
typedef struct mp_update_plan mp_update_plan; /* device table over the tensors of an update */

/* Loss-scale policy (Section 3.1, item 1).  dynamic != 0: halve S (not below min_scale) after
 * a step whose gradients held an inf/NaN, double it (not above max_scale) after
 * growth_interval clean steps in a row.  dynamic == 0: S stays init_scale (static loss
 * scaling); an overflow step is still skipped.
 * overflow_tolerance = H > 1 selects a second policy that the paper does not describe: S is
 * halved at the H-th overflow since S last changed (a doubling clears the count too), so an
 * isolated overflow costs a skipped step but no halving.  Every overflow step is still
 * skipped and still restarts the run of clean steps.  H = 1 is the plain rule. */
typedef struct {
  float init_scale;        /* > 0 */
  float min_scale;         /* > 0 */
  float max_scale;         /* >= min_scale */
  int32_t growth_interval; /* >= 1 */
  int32_t dynamic;
  int32_t overflow_tolerance; /* >= 1 */
} mp_scaler_config;

typedef enum { MP_OPT_ADAM = 0, MP_OPT_MOMENTUM = 1 } mp_opt_kind;

/* Optimizer run on the FP32 master (Section 3.2).  Adam: m = b1 m + (1-b1) g,
 * v = b2 v + (1-b2) g^2, w -= lr (m/(1-b1^t)) / (sqrt(v/(1-b2^t)) + eps), t = number of
 * applied steps including this one.  Momentum: u = mu u + g, w -= lr u.
 * weight_decay adds weight_decay * w32 to g before the moments (Section 3.3). */
typedef struct {
  int32_t kind; /* mp_opt_kind */
  float lr, beta1, beta2, eps, momentum, weight_decay;
} mp_optim_config;

/* Host copy of the device state, filled by mp_state_read. */
typedef struct {
  float scale;         /* S that the NEXT step will use                                     */
  float min_scale, max_scale;
  int32_t growth_interval, dynamic;
  int32_t good_steps;  /* clean steps since S last changed                                  */
  int32_t found_inf;   /* flag accumulated by the current step so far                       */
  int32_t status;      /* MP_OK or the first device-side error (MP_ERR_TIMEOUT, or
                          MP_ERR_INVALID_ARG for a token id out of range), see above        */
  int32_t overflow_tolerance;
  int32_t strikes;     /* overflows since S last changed (dynamic scale with tolerance 1:
                          always 0; static scale: S never changes, so every overflow counts) */
  int64_t t;           /* applied optimizer steps                                           */
  int64_t step;        /* all steps                                                         */
  int64_t skipped;     /* overflow steps                                                    */
} mp_state_host;

/* One record per mp_loss_scale_update call, kept in a device ring of MP_LOG_CAPACITY. */
typedef struct {
  int64_t step;
  int64_t t;           /* after the step */
  float scale_before, scale_after;
  int32_t found_inf, good_steps;
} mp_log_record;
#define MP_LOG_CAPACITY 4096

/* ---- the five calls of the step ------------------------------------------------------ */

/* Forward product (Section 3.1): Y[M,N] = rn16( sum_k X[m,k] * W[k,n] ), FP32 accumulation.
 * X16 [M,K] ldx>=K, W16 [K,N] ldw>=N, Y16 [M,N] ldy>=N, all FP16 device buffers.
 * workspace: device scratch of at least mp_gemm_workspace_bytes(M,K,N,MP_OP_FWD) bytes
 * (may be NULL when that is 0).  Errors: INVALID_ARG, ALIGNMENT, NOMEM (workspace too
 * small), UNSUPPORTED_ARCH, CUDA. */
int mp_linear_fwd(const void* X16, int64_t ldx, const void* W16, int64_t ldw, void* Y16,
                  int64_t ldy, int64_t M, int64_t K, int64_t N, void* workspace,
                  size_t workspace_bytes, void* stream);

/* Data gradient (Section 3.2, "gradients are in FP16"): dX[M,K] = rn16( sum_n dY[m,n] *
 * W[k,n] ).  W is read in place as stored (no transposed copy). */
int mp_linear_bwd_dgrad(const void* dY16, int64_t lddy, const void* W16, int64_t ldw,
                        void* dX16, int64_t lddx, int64_t M, int64_t K, int64_t N,
                        void* workspace, size_t workspace_bytes, void* stream);

/* Weight gradient: dW[K,N] = rn16( sum_m X[m,k] * dY[m,n] ), still multiplied by S.
 * If state != NULL, state->found_inf is set when any element written to dW16 is inf or NaN
 * (the gradient inspection of Section 3.1, item 1, done where the gradient is produced). */
int mp_linear_bwd_wgrad(const void* X16, int64_t ldx, const void* dY16, int64_t lddy,
                        void* dW16, int64_t lddw, int64_t M, int64_t K, int64_t N,
                        mp_state* state, void* workspace, size_t workspace_bytes, void* stream);

/* Fused master update over every tensor of the plan (Section 3.2): if the step's flag is
 * clear, g = float(g16) * (1/S), optimizer on w32 (and m, v), w16 = rn16(w32); if it is set,
 * nothing is written.  check_mode 0: trust state->found_inf as set by the wgrad calls;
 * check_mode 1: first inspect every g16 of the plan (sets state->found_inf), then update.
 * S, t and the flag are read on the device; nothing returns to the host. */
int mp_master_update(mp_update_plan* plan, mp_state* state, const mp_optim_config* opt,
                     int check_mode, void* stream);

/* Loss-scale state machine (Section 3.1, item 1: the scale for the next step is chosen from
 * this step's inspection).  Flag set: S = max(S/2, min_scale), good = 0, skipped++.
 * Flag clear: t++, good++, and when good == growth_interval: S = min(2S, max_scale), good = 0.
 * Then the flag is cleared, step++ and a log record is appended.  One tiny kernel. */
int mp_loss_scale_update(mp_state* state, void* stream);

/* Weight gradient for callers that must not allocate.  (The paper has no counterpart: this is
 * a packaging variant of mp_linear_bwd_wgrad, same arithmetic, same results bit for bit.)
 *
 * Who needs it: code that runs where device allocation is off the table -- a training or
 * serving runtime that has already handed all free device memory to its own pool, so that a
 * cudaMalloc would fail; a step that must not hit the implicit device-wide synchronisation an
 * allocation or free causes; a plugin whose host forbids allocator calls inside its callbacks.
 * Such callers also may have no spare buffer to lend as `workspace`.
 *
 * Differences from mp_linear_bwd_wgrad: there is no workspace argument.  The split-reduction
 * scratch is an array built into the library image, MP_STATIC_SCRATCH_BYTES (32 MiB) per GPU,
 * reserved on every GPU that loads the library until the process exits.  Sizes whose scratch
 * need (mp_gemm_workspace_bytes(M,K,N,MP_OP_WGRAD)) exceeds it are refused with
 * MP_ERR_TOO_LARGE and nothing is launched.  The call makes no cudaMalloc/cudaFree and uses no
 * allocating library routine.
 *
 * The first call on each device looks up the array's device address (one cheap runtime query,
 * no allocation, done with that device current), and like every product call the first one per
 * device and kernel flavour also sets kernel attributes and asks for occupancy; make a first
 * call with sizes of the same class (K above or at most 128, i.e. the same kernel flavour)
 * before starting any stream capture.  All calls on a device share the one array: two calls whose kernels may
 * overlap on the GPU (different streams) race on it and must be ordered by the caller.  The
 * array keeps whatever the previous call left; that is harmless because each call overwrites
 * every partial sum it later reads, so nothing has to start at zero. */
#define MP_STATIC_SCRATCH_BYTES (32u << 20)
int mp_linear_bwd_wgrad_static(const void* X16, int64_t ldx, const void* dY16, int64_t lddy,
                               void* dW16, int64_t lddw, int64_t M, int64_t K, int64_t N,
                               mp_state* state, void* stream);
/* Size of that built-in scratch in bytes (equals MP_STATIC_SCRATCH_BYTES). */
size_t mp_static_scratch_bytes(void);

/* ---- several independent layers of one shape in one launch ------------------------------
 * The products of Section 3.1 for `count` (1 .. mp_max_group()) layers that have the same M, K,
 * N and leading dimensions and do not depend on one another (the query, key and value
 * projections of an attention block; the per-layer gate products of a stack whose layers are
 * fed independently).  X16, W16, Y16 ... are host arrays of `count` device pointers; each
 * problem obeys the rules of the single call of the same name and gets that call's result (bit
 * for bit when both split the reduction the same way; otherwise the FP32 partial sums are added
 * in another, equally fixed order).  One launch walks the tiles of all problems, so a product too small to fill
 * the GPU's waves on its own does not leave SMs idle.  workspace: at least
 * mp_gemm_workspace_bytes_grouped(count, M, K, N, op) bytes.  Errors as for the single calls;
 * INVALID_ARG also for count outside 1 .. mp_max_group(). */
int mp_linear_fwd_grouped(int count, const void* const* X16, int64_t ldx, const void* const* W16,
                          int64_t ldw, void* const* Y16, int64_t ldy, int64_t M, int64_t K, int64_t N,
                          void* workspace, size_t workspace_bytes, void* stream);
int mp_linear_bwd_dgrad_grouped(int count, const void* const* dY16, int64_t lddy, const void* const* W16,
                                int64_t ldw, void* const* dX16, int64_t lddx, int64_t M, int64_t K,
                                int64_t N, void* workspace, size_t workspace_bytes, void* stream);
/* ORs "an inf or NaN was stored" of every problem into state->found_inf (state may be NULL). */
int mp_linear_bwd_wgrad_grouped(int count, const void* const* X16, int64_t ldx, const void* const* dY16,
                                int64_t lddy, void* const* dW16, int64_t lddw, int64_t M, int64_t K,
                                int64_t N, mp_state* state, void* workspace, size_t workspace_bytes,
                                void* stream);
/* The grouped forward product with the bias and activation of mp_linear_fwd_act: bias16 is a
 * host array of `count` device pointers (or NULL for no bias), one activation for all. */
int mp_linear_fwd_act_grouped(int count, const void* const* X16, int64_t ldx, const void* const* W16,
                              int64_t ldw, const void* const* bias16, void* const* Y16, int64_t ldy,
                              int64_t M, int64_t K, int64_t N, int act, float clip, void* workspace,
                              size_t workspace_bytes, void* stream);
/* Largest `count` the grouped calls take. */
int mp_max_group(void);

/* ---- layers with a bias and an activation ------------------------------------------------
 * The models of the paper's Section 5 follow their dense products with a bias and a
 * nonlinearity (ReLU in the Transformer feed-forward block, clipped ReLU in DeepSpeech2).  The
 * paper gives no arithmetic for them; this library's reading: the FP16 bias is added to the
 * FP32 sum before the single rounding to FP16, the activation acts on that FP32 value, and the
 * backward pass zeroes the FP16 data gradient where the stored FP16 output of the activated
 * layer is outside the activation's linear range. */
typedef enum { MP_ACT_NONE = 0, MP_ACT_RELU = 1, MP_ACT_CLIPPED_RELU = 2 } mp_activation;

/* Y[M,N] = rn16( act( sum_k X[m,k] W[k,n] + bias[n] ) ).  bias16: N FP16 values, 16-byte aligned,
 * or NULL.  act: mp_activation; clip: upper bound of MP_ACT_CLIPPED_RELU (min(max(x,0),clip)).
 * Other arguments and errors as mp_linear_fwd. */
int mp_linear_fwd_act(const void* X16, int64_t ldx, const void* W16, int64_t ldw, const void* bias16,
                      void* Y16, int64_t ldy, int64_t M, int64_t K, int64_t N, int act, float clip,
                      void* workspace, size_t workspace_bytes, void* stream);

/* dX[m,k] = rn16( sum_n dY[m,n] W[k,n] ) where A[m,k] passes the activation (A > 0 for ReLU,
 * 0 < A < clip for clipped ReLU), else +0.  A16 [M,K] (lda >= K) is this layer's input, i.e.
 * the activated FP16 output of the layer below; it may alias nothing that is written.  With
 * MP_ACT_NONE the call equals mp_linear_bwd_dgrad and A16 may be NULL. */
int mp_linear_bwd_dgrad_act(const void* dY16, int64_t lddy, const void* W16, int64_t ldw,
                            const void* A16, int64_t lda, void* dX16, int64_t lddx, int64_t M,
                            int64_t K, int64_t N, int act, float clip, void* workspace,
                            size_t workspace_bytes, void* stream);

/* db[n] = rn16( sum_m dY[m,n] ), FP32 accumulation in a fixed order (results do not depend on
 * timing), still multiplied by S.  Sets state->found_inf if a stored value is inf or NaN (state
 * may be NULL).  workspace: at least mp_bias_grad_workspace_bytes(M,N) bytes of device scratch. */
int mp_bias_grad(const void* dY16, int64_t lddy, void* db16, int64_t M, int64_t N, mp_state* state,
                 void* workspace, size_t workspace_bytes, void* stream);
size_t mp_bias_grad_workspace_bytes(int64_t M, int64_t N);
/* The same for `count` (1 .. mp_max_group()) gradients of one shape and row pitch in one pair of launches: dY16 and
 * db16 are host arrays of `count` device pointers; every result is the single call's, bit for bit.
 * workspace: at least count * mp_bias_grad_workspace_bytes(M,N) bytes. */
int mp_bias_grad_grouped(int count, const void* const* dY16, int64_t lddy, void* const* db16, int64_t M,
                         int64_t N, mp_state* state, void* workspace, size_t workspace_bytes, void* stream);

/* LSTM cell for a gate product G = [x;h] W of 4H columns in the order i, f, g, o (the GNMT-like
 * layers of Section 5; the paper gives no arithmetic, so: FP16 gates and states in memory, the
 * cell evaluated in FP32 with sigma(x) = 1/(1+exp(-x)) and tanh, one rounding per output).
 *   c_new = sigma(f) c_prev + sigma(i) tanh(g),   h = sigma(o) tanh(c_new)
 * G16 [M,4H] with ldg >= 4H; c_prev16, c_new16, h16 dense [M,H]; H and ldg multiples of 8. */
int mp_lstm_cell_fwd(const void* G16, int64_t ldg, const void* c_prev16, void* c_new16, void* h16,
                     int64_t M, int64_t H, void* stream);

/* Backward of the cell from the stored FP16 gates and states: dh16 is the gradient at h,
 * dc_in16 the gradient arriving at c_new from the next time step (NULL = none).  Writes dG16
 * [M,4H] (gradient at the gate pre-activations, the dY of the gate product's backward calls)
 * and dc_prev16 [M,H]; tanh(c_new) is taken from the stored FP16 c_new.  Gradients stay
 * multiplied by the loss scale. */
int mp_lstm_cell_bwd(const void* G16, int64_t ldg, const void* c_prev16, const void* c_new16,
                     const void* dh16, const void* dc_in16, void* dG16, int64_t lddg, void* dc_prev16,
                     int64_t M, int64_t H, void* stream);

/* ---- operators of a token model ---------------------------------------------------------
 * What stands around the products when the stack is a language model: the embedding that turns
 * tokens into its input, the norms, gate and residual sum that join its blocks, the loss whose
 * gradient enters its top layer, and an AdamW update.  (The paper's models have an embedding and
 * train with Adam; it gives no arithmetic for these.)  Matrices are FP16 with row pitches that
 * are multiples of 8 and may have any width: what lies between the width and the pitch is not
 * written, and its values do not matter.  Rows and vectors of gains or gates are read in whole units
 * of 16 bytes: what follows the last element inside its unit is read too, and dropped.  Sums, norms and softmax statistics are FP32; each
 * stored value is rounded once.  No call uses floating-point atomics: the same inputs give the
 * same bits.  Gradients arrive and leave multiplied by the loss scale; a call that is given a
 * state sets state->found_inf when a parameter gradient or logit gradient that it stores is inf
 * or NaN. */

/* Y[i,:] = rn16( scale * W[ids[i],:] ), and +0 where ids[i] == pad_id (pad_id < 0: no padding id).
 * ids: n integers of id_bytes (4 or 8) bytes each, aligned to id_bytes; W16 [V,D] ldw >= D, Y16
 * [n,D] ldy >= D.  A row whose id is neither the padding id nor in 0 .. V-1 becomes NaN, and
 * state->status (state may be NULL) becomes MP_ERR_INVALID_ARG.  n = 0 is legal. */
int mp_embedding_fwd(const void* ids, int id_bytes, const void* W16, int64_t ldw, void* Y16, int64_t ldy,
                     int64_t n, int64_t V, int64_t D, int64_t pad_id, float scale, mp_state* state,
                     void* stream);

/* Gradient of the lookup: dW[v,:] = rn16( scale * sum_{i: ids[i] = v} dY[i,:] ) for every v of
 * 0 .. V-1; rows of the padding id and of ids that do not occur become +0.  The tokens are sorted
 * by id, in ascending i for each id, and the sums follow that order in FP32 (a long run of one id
 * as the sums of its pieces, in order).  An id out of range adds to nothing and sets state->status as above.
 * workspace: at least mp_embedding_bwd_workspace_bytes(n,V,D) bytes of device scratch, 16-byte
 * aligned.  n below 2^31 - 129, V below 2^31 - 1. */
int mp_embedding_bwd(const void* ids, int id_bytes, const void* dY16, int64_t lddy, void* dW16, int64_t ldw,
                     int64_t n, int64_t V, int64_t D, int64_t pad_id, float scale, mp_state* state,
                     void* workspace, size_t workspace_bytes, void* stream);
size_t mp_embedding_bwd_workspace_bytes(int64_t n, int64_t V, int64_t D);

/* Norms before and after a block, with the block's gate and the residual scale, for rows of D
 * elements (1 .. MP_NORM_MAX_D).  With y the block's output:
 *   h = norm(y) * g_post,   x_out = res_scale * x + gate * h,   n = norm(x_out) * g_pre
 * norm(v) = v / sqrt(mean(v^2) + eps) for MP_NORM_RMS, (v - mean(v)) / sqrt(var(v) + eps) for
 * MP_NORM_LAYER.  n, the next block's input, is formed from the FP32 x_out before its rounding.
 * x, x_out: the residual stream, FP16 (x_bytes 2, pitch a multiple of 8) or FP32 (x_bytes 4, pitch
 * a multiple of 4).  gate16: NULL (1), one vector of D for all rows (ldgate 0), or a matrix [M,D]
 * (ldgate >= D).  stats (may be NULL): M records of four FP32 values, mean and 1/sqrt of y's norm
 * and of x_out's (means 0 for MP_NORM_RMS), for the backward call.
 * g_post16 NULL: the norm before the first block alone, n = norm(x) * g_pre; y16, x_out and gate16
 * must be NULL, and the first two values of a record are 0.  M = 0 is legal.
 * x_out may be x itself, n16 may be y16 itself (same pitch). */
typedef enum { MP_NORM_RMS = 0, MP_NORM_LAYER = 1 } mp_norm_kind;
#define MP_NORM_MAX_D 16384
int mp_block_norm_fwd(int kind, float eps, float res_scale, const void* x, int x_bytes, int64_t ldx,
                      const void* y16, int64_t ldy, const void* g_post16, const void* gate16, int64_t ldgate,
                      void* x_out, int64_t ldxo, const void* g_pre16, void* n16, int64_t ldn, float* stats,
                      int64_t M, int64_t D, void* stream);

/* Backward of the call above, from the stored x_out, y and stats.  dn16: gradient at n; dx_out:
 * gradient that reaches x_out from above (of x's type; NULL = none).  With xhat, yhat the normed rows:
 *   gx = dx_out + d norm(x_out)/d x_out applied to dn * g_pre,   dx = res_scale * gx,
 *   dy = d norm(y)/d y applied to gx * gate * g_post,
 *   dg_pre = sum_rows dn * xhat,   dg_post = sum_rows gx * gate * yhat,
 *   dgate = gx * h, summed over the rows for a gate vector, [M,D] (lddgate >= D) for a gate matrix.
 * With g_post16 NULL: dx = gx, and y16, dy16, gate16, dg_post16, dgate16 must be NULL; dgate16 is
 * NULL exactly when gate16 is.  dx may be dx_out or x_out itself, dy16 may be dn16 or y16 itself, a gate
 * matrix's dgate16 may be gate16 itself (same pitch).  The gradients of the gains and of a gate
 * vector are FP32 sums over the rows in a fixed order.  workspace: at least
 * mp_block_norm_bwd_workspace_bytes(M,D) bytes, 16-byte aligned. */
int mp_block_norm_bwd(int kind, float res_scale, const void* dn16, int64_t lddn, const void* dx_out,
                      int64_t lddxo, const void* x_out, int x_bytes, int64_t ldxo, const void* y16, int64_t ldy,
                      const void* g_post16, const void* gate16, int64_t ldgate, const void* g_pre16,
                      const float* stats, void* dx, int64_t lddx, void* dy16, int64_t lddy, void* dg_post16,
                      void* dgate16, int64_t lddgate, void* dg_pre16, int64_t M, int64_t D, mp_state* state,
                      void* workspace, size_t workspace_bytes, void* stream);
size_t mp_block_norm_bwd_workspace_bytes(int64_t M, int64_t D);

/* Clipped policy loss with a KL term, forward and backward in one call.  For row i with logits z,
 * target t and weight w:
 *   lp = z_t - log sum_j exp(z_j),   r = exp(lp - old_logp),   d = ref_logp - lp
 *   l  = -min( r A, clip(r, 1 - clip_lo, 1 + clip_hi) A ) + kl_coef (exp(d) - d - 1)
 *   dz_j = rn16( grad_scale * S * w * dl/dlp * ([j = t] - exp(z_j) / sum exp(z)) )
 * S: the loss scale of `state` (1 without a state).  Where r A equals its clipped value the gradient is
 * that of r A.  logp[i] = lp, token_loss[i] = w l, loss[0] = sum_i token_loss[i] (fixed order; may be
 * NULL).  A row of weight 0 is masked: nothing of it is read, its outputs are 0.  ref_logp NULL or
 * kl_coef 0: no KL term.  A target outside 0 .. V-1 in a row that is not masked gives NaN for the row's outputs
 * and sets state->status.  logits16 [N,V] ldl >= V, dlogits16 [N,V] lddl >= V; dlogits16 may be
 * logits16 itself (same pitch), or NULL for the forward pass alone.  targets: N integers of id_bytes
 * (4 or 8) bytes.  N = 0 is legal (loss 0).  V is at most MP_POLICY_MAX_V. */
#define MP_POLICY_MAX_V 524288
typedef struct {
  float clip_lo, clip_hi; /* 0 <= clip_lo, 0 <= clip_hi */
  float kl_coef;
  float grad_scale;
} mp_policy_config;
int mp_policy_loss(const void* logits16, int64_t ldl, const void* targets, int id_bytes, const float* old_logp,
                   const float* ref_logp, const float* advantage, const float* weight, int64_t N, int64_t V,
                   const mp_policy_config* cfg, void* dlogits16, int64_t lddl, float* logp, float* token_loss,
                   float* loss, mp_state* state, void* stream);

/* logp[i] = z_t - log sum_j exp(z_j): what the loss takes as old_logp and ref_logp.  weight: rows
 * of weight 0 give 0 and are not read (NULL: every row counts).  Other arguments as above; without
 * a state an id out of range shows as NaN alone. */
int mp_token_logp(const void* logits16, int64_t ldl, const void* targets, int id_bytes, const float* weight,
                  int64_t N, int64_t V, float* logp, mp_state* state, void* stream);

/* Token scores: for row i with logits z and x = z / temperature, lp_j = x_j - log sum_l exp(x_l),
 *   logp[i] = lp at targets[i],   entropy[i] = -sum_j exp(lp_j) lp_j,
 *   top_ids[i, 0 .. k-1], top_logp[i, ..] = the k largest logits' ids and lp, largest first; of equal logits the
 *   lower id comes first.  The same call gives the same bits; the last bits of a row's values may differ with
 *   N, by how many blocks share a row.
 * targets: N integers of id_bytes (4 or 8) bytes; targets and logp are both given or both NULL.  entropy and weight may be
 * NULL.  top_ids (int32) and top_logp [N, k] dense, 1 <= k <= min(V, MP_TOP_MAX_K).  A row of weight 0 is not
 * read: its ids become -1, its values 0.  A target out of range gives NaN and a status, as in mp_policy_loss.
 * A row with +inf or NaN among its logits has NaN for its values; its ids are then not specified (-1 or a
 * token).  temperature: MP_MIN_TEMPERATURE .. MP_MAX_TEMPERATURE. */
#define MP_TOP_MAX_K 128
#define MP_MIN_TEMPERATURE 1e-3f
#define MP_MAX_TEMPERATURE 1e3f
int mp_token_top(const void* logits16, int64_t ldl, const void* targets, int id_bytes, const float* weight, int64_t N,
                 int64_t V, int64_t k, float temperature, float* logp, float* entropy, int32_t* top_ids,
                 float* top_logp, mp_state* state, void* stream);

/* Distillation from a teacher's top entries, forward and backward in one call.  ids, teacher_logp [N, K] dense: the tokens
 * that the teacher lists for a row and their log-probabilities a (as mp_token_top gives them, at the same
 * temperature); an id of -1 is no entry.  With lq the student's log-probabilities at the temperature:
 *   tail 1:  l = sum_e p_e (a_e - lq_e) + r (log r - log sum_{j not listed} exp(lq_j)),  p = exp(a), r = max(0, 1 - sum_e p_e)
 *   tail 0:  l = sum_e p_e (log p_e - lq_e),  p = the softmax of a over the row's entries (top logits / temperature do as well)
 *   token_loss[i] = w l,   loss[0] = sum_i token_loss[i] (fixed order; may be NULL)
 *   dz_j = rn16( grad_scale * S * w * dl/dz_j )
 * An entry of probability 0 adds nothing.  Without an unlisted token of finite logit r is 0.  A row of weight 0 is
 * masked as in mp_policy_loss.  An id that is out of range, or that a row lists twice (and whose logit is
 * not -inf), gives NaN for the row's outputs and sets state->status.  logits16, dlogits16, S, N = 0 and the limits of V as in
 * mp_policy_loss; 1 <= K <= min(V, MP_DISTILL_MAX_K). */
#define MP_DISTILL_MAX_K 128
typedef struct {
  float temperature;
  int32_t tail;
  float grad_scale;
} mp_distill_config;
int mp_distill_loss(const void* logits16, int64_t ldl, const void* ids, int id_bytes, const float* teacher_logp,
                    int64_t K, const float* weight, int64_t N, int64_t V, const mp_distill_config* cfg,
                    void* dlogits16, int64_t lddl, float* token_loss, float* loss, mp_state* state, void* stream);

/* AdamW (weight decay apart from the gradient) over the tensors of a plan, on the FP32 master, with
 * the flag, S and t of `state` as in mp_master_update.  Per element, with g = float(g16) / S,
 * c1 = 1 - beta1^t, c2 = 1 - beta2^t:
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,   r = sqrt(v)
 *   w = w - (lr weight_decay decay[i]) w,   w = w - (lr / c1) ( m / (r / sqrt(c2) + eps) ),   w16 = rn16(w)
 * decay[i]: factor of tensor i (0 for the gains and biases that should not decay).
 * state_bits 32: m[i], v[i] are FP32 buffers of count[i].  state_bits 8: m[i], v[i] are bytes that
 * hold E4M3 numbers, of m and of r, each to be multiplied by the FP32 scale of its block of
 * MP_ADAMW_BLOCK elements (m_scale[i], v_scale[i]: ceil(count[i] / MP_ADAMW_BLOCK) values); the
 * block's scale is its largest magnitude / 448 (0 when that is below 2^-100: the block is stored as
 * zeros).  r is kept instead of v because its range is half as many binades; an r above 0 is stored
 * as at least the smallest number above 0, since a step by m / (0 + eps) would be far too long.
 * All-zero buffers and scales are the initial state.  Errors as mp_update_plan_create and mp_master_update. */
typedef struct {
  double lr, beta1, beta2, eps, weight_decay; /* 1 - beta is formed in double before it is rounded */
} mp_adamw_config;
#define MP_ADAMW_BLOCK 256
typedef struct mp_adamw_plan mp_adamw_plan;
int mp_adamw_plan_create(int n, void* const* g16, void* const* w32, void* const* m, void* const* v,
                         void* const* w16, const int64_t* count, const float* decay, int state_bits,
                         float* const* m_scale, float* const* v_scale, mp_adamw_plan** out);
int mp_adamw_plan_destroy(mp_adamw_plan* plan); /* NULL is accepted */
int mp_adamw_update(mp_adamw_plan* plan, mp_state* state, const mp_adamw_config* opt, int check_mode,
                    void* stream);

/* Norms of queries and keys for each head, and the position rotation, in one pass.  A row of x16 holds q_heads
 * query heads and then k_heads key heads of D elements each (D a multiple of 8, at most MP_HEAD_MAX_D; what
 * follows in the row, values for instance, is left alone).  Each head u becomes
 *   n = u / sqrt(mean(u^2) + eps) * g,   y = R n
 * with g = gq16 for query heads, gk16 for key heads (D elements each; both NULL: 1).  R turns the first rot
 * elements (a multiple of 16, 0: none) pair by pair: for pair i with angle t = positions[row] freqs[i]
 *   (a, b) -> (a cos t - b sin t, a sin t + b cos t)
 * pairs are elements (i, i + rot / 2) with pairs 0, (2 i, 2 i + 1) with pairs 1.  positions: T integers of
 * pos_bytes (4 or 8) bytes, of any size; freqs: rot / 2 FP64 values in radians, finite.  The angle is formed in 64-bit fixed
 * point turns, so far positions keep their precision.  eps >= 0; with 0 a head of zeros has no norm and gives NaN.  y16 may be x16
 * itself (same pitch).  T = 0 is legal. */
#define MP_HEAD_MAX_D 256
int mp_head_norm_rope_fwd(const void* x16, int64_t ldx, const void* gq16, const void* gk16, const void* positions,
                          int pos_bytes, const double* freqs, int64_t rot, int pairs, float eps, void* y16,
                          int64_t ldy, int64_t T, int64_t q_heads, int64_t k_heads, int64_t D, void* stream);

/* Backward of the call above, from its input x16: with u = R^-1 dy and xhat the normed head before the gain,
 *   dx = (u g - xhat mean(u g xhat)) / sqrt(mean(x^2) + eps),   dg = sum over rows and heads of u xhat
 * dx16 may be dy16 or x16 itself (same pitch).  dgq16, dgk16: D elements each, NULL exactly when the gains are;
 * FP32 sums in a fixed order, rounded once.  workspace: at least mp_head_norm_rope_bwd_workspace_bytes(..) bytes,
 * 16-byte aligned (none needed without gains). */
int mp_head_norm_rope_bwd(const void* dy16, int64_t lddy, const void* x16, int64_t ldx, const void* gq16,
                          const void* gk16, const void* positions, int pos_bytes, const double* freqs, int64_t rot,
                          int pairs, float eps, void* dx16, int64_t lddx, void* dgq16, void* dgk16, int64_t T,
                          int64_t q_heads, int64_t k_heads, int64_t D, mp_state* state, void* workspace,
                          size_t workspace_bytes, void* stream);
size_t mp_head_norm_rope_bwd_workspace_bytes(int64_t T, int64_t q_heads, int64_t k_heads, int64_t D);

/* Attention over packed sequences, for each of `heads` heads of D elements (a multiple of 8, at most
 * MP_ATTENTION_MAX_D):
 *   s_ij = scale q_i . k_j,   p_ij = exp(s_ij - lse_i),   lse_i = log sum_j exp(s_ij),   o_i = sum_j p_ij v_j
 * over the keys j of the query's own sequence that it sees: all of them; with causal 1 those with
 * j <= i; with a window (causal only; 0: none) those of them with i - j < window.  Head h of a row
 * is its elements h D .. (h + 1) D - 1; query head h reads key head h kv_heads / heads (kv_heads
 * divides heads).  q16, o16 [T, heads D], k16, v16 [T, kv_heads D] with pitches of their own, so they may be
 * columns of one product.  lse [heads, T] FP32.  offsets: n_seq + 1 integers of id_bytes (4 or 8)
 * bytes in device memory, ascending within 0 .. T: sequence b is rows offsets[b] .. offsets[b + 1] - 1
 * (none when they are equal); rows of no sequence are not read, and their outputs stay as they were.
 * Offsets out of order or range give status MP_ERR_INVALID_ARG in the state, and which sequences are worked
 * on is then not specified (nothing outside the matrices is touched).  Scores, sums and outputs
 * are FP32 until one rounding; the weights p enter their product in FP16 times a power of two: those down to 2^-21 of their row's
 * largest keep all its bits, smaller ones are off by at most 2^-32 of the largest.  Values of other sequences never matter;
 * inf or NaN in a key or value may reach all queries of its own sequence, those that do not see it
 * too.  o16 may not be an input (refused where their addresses are equal).  T = 0 or n_seq = 0 is legal.  scale > 0. */
#define MP_ATTENTION_MAX_D 128
#define MP_ATTENTION_MAX_ROWS (1 << 30)
int mp_attention_fwd(const void* q16, int64_t ldq, const void* k16, int64_t ldk, const void* v16, int64_t ldv,
                     void* o16, int64_t ldo, float* lse, const void* offsets, int id_bytes, int64_t n_seq,
                     int64_t T, int64_t heads, int64_t kv_heads, int64_t D, float scale, int causal,
                     int64_t window, mp_state* state, void* stream);

/* Backward of the call above, from its inputs, o16 and lse; do16 [T, heads D]: gradient at o.  With
 * delta_i = do_i . o_i and ds_ij = p_ij (do_i . v_j - delta_i):
 *   dv_j = sum_i p_ij do_i,   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i
 * (for a key head summed over the query heads that share it).  p and ds enter their products in FP16: p times 2^12, so weights
 * down to 2^-26 keep all its bits, and ds times a power of two that fits the largest rows of do and v, so the loss scale costs
 * none.  p is formed again from s - lse in FP32: with scores of about 2^k it is off by some 2^(k - 22) of itself, and from 2^23
 * on it may pass FP16's range (inf or NaN in the gradients of those rows' sequences).  Every sum runs in a fixed order.  Rows of
 * no sequence are not read, and their gradients stay as they were.  dq16 [T, heads D], dk16, dv16 [T, kv_heads D] may not be
 * inputs or one another.  inf or NaN in a row of do16 or v16 may reach all gradients of its sequence, and the other sequences'
 * ds then goes without that power of two.  workspace: at least mp_attention_bwd_workspace_bytes(..) bytes of device scratch,
 * 16-byte aligned. */
int mp_attention_bwd(const void* do16, int64_t lddo, const void* q16, int64_t ldq, const void* k16, int64_t ldk,
                     const void* v16, int64_t ldv, const void* o16, int64_t ldo, const float* lse, void* dq16,
                     int64_t lddq, void* dk16, int64_t lddk, void* dv16, int64_t lddv, const void* offsets,
                     int id_bytes, int64_t n_seq, int64_t T, int64_t heads, int64_t kv_heads, int64_t D, float scale,
                     int causal, int64_t window, mp_state* state, void* workspace, size_t workspace_bytes,
                     void* stream);
size_t mp_attention_bwd_workspace_bytes(int64_t T, int64_t heads, int64_t kv_heads, int64_t D);

/* ---- auxiliaries --------------------------------------------------------------------- */

enum { MP_OP_FWD = 0, MP_OP_DGRAD = 1, MP_OP_WGRAD = 2 };

/* Scratch bytes the GEMM of `op` needs for these sizes (0 when it needs none). */
size_t mp_gemm_workspace_bytes(int64_t M, int64_t K, int64_t N, int op);
/* The same for a grouped call over `count` problems (0 for a count the calls refuse). */
size_t mp_gemm_workspace_bytes_grouped(int count, int64_t M, int64_t K, int64_t N, int op);

/* dY16[i] = rn16( S * g32[i] ), S read from the device state (Section 3.1, item 1: the loss
 * is scaled; for a linear stack that is the gradient entering the top layer). */
int mp_scale_upstream(const float* g32, void* dY16, int64_t n, const mp_state* state,
                      void* stream);

/* Sets state->found_inf if any of the n FP16 values at g16 is inf or NaN. */
int mp_check_finite(const void* g16, int64_t n, mp_state* state, void* stream);

int mp_state_create(const mp_scaler_config* cfg, mp_state** out);
int mp_state_destroy(mp_state* state); /* NULL is accepted */
/* Synchronises `stream`, then copies the device state to *out. */
int mp_state_read(mp_state* state, mp_state_host* out, void* stream);
/* Overwrites the device state (resume from a checkpoint); synchronises `stream`. */
int mp_state_write(mp_state* state, const mp_state_host* in, void* stream);
/* Copies up to max_records of the most recent log records, oldest first, to out (host);
 * *n_out receives the count.  Synchronises `stream`. */
int mp_state_read_log(mp_state* state, mp_log_record* out, int max_records, int* n_out,
                      void* stream);

/* Data-parallel runs whose ranks each inspect only a slice of the summed gradients (Section 4
 * of the paper: replicas that exchange gradients; the sharded-update schedule) agree on the
 * overflow flag by reducing one word across ranks.  These two calls move the flag between the
 * device state and a caller-owned int32 device word, asynchronously on `stream`, with no host
 * round trip: export writes *word = (found_inf != 0); import ORs (*word != 0) into found_inf.
 * word: device pointer, 4-byte aligned. */
int mp_state_export_flag(const mp_state* state, int32_t* word, void* stream);
int mp_state_import_flag(mp_state* state, const int32_t* word, void* stream);

/* Plan over n tensors: g16[i], w16[i] FP16 and w32[i], m[i], v[i] FP32 device buffers of
 * count[i] elements each (count[i] == 0 is legal and skipped).  v may be NULL for a plan
 * used only with momentum (m then holds the momentum buffer).  The pointer arrays are host
 * arrays and are copied; the tensors stay the caller's. */
int mp_update_plan_create(int n, void* const* g16, void* const* w32, void* const* m,
                          void* const* v, void* const* w16, const int64_t* count,
                          mp_update_plan** out);
int mp_update_plan_destroy(mp_update_plan* plan); /* NULL is accepted */

/* Error-path self-test (not one of the step's calls; the paper has no counterpart).  Launches
 * the forward product's kernel on ONE output tile (M <= 128, N <= 256; arguments otherwise as
 * mp_linear_fwd) with its loader told to fetch nothing and every pipeline wait limited to
 * wait_us microseconds (1 .. 2000000).  No copy is ever in flight: the waits run out, the
 * kernel records MP_ERR_TIMEOUT (device-wide and, if state != NULL, in state->status), frees
 * its tensor memory and returns without writing Y16.  It exists so that the library's
 * reaction to an expired wait can be exercised on a healthy GPU. */
int mp_selftest_wait_timeout(const void* X16, int64_t ldx, const void* W16, int64_t ldw, void* Y16,
                             int64_t ldy, int64_t M, int64_t K, int64_t N, int64_t wait_us,
                             mp_state* state, void* stream);

/* Synchronises the device and reports in *out the first device-side error recorded by a GEMM
 * kernel since the last call (MP_OK, or MP_ERR_TIMEOUT when a bounded wait on a pipeline
 * barrier expired; the kernel then skipped its remaining work and returned).  Clears it. */
int mp_gemm_device_status(int* out);

/* Message of the last error on the calling thread ("" if none). */
const char* mp_last_error(void);

/* Number of kernels this library has launched in the calling process (for accounting). */
int64_t mp_kernel_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* MP_H_ */
