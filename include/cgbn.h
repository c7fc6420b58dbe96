/*
 * libcgbn -- Cross-GPU Batch Normalization (CGBN) forward and backward for one
 * MI355X (gfx950), with the method's n devices appearing as K "virtual
 * devices": K contiguous, equal sub-batch shards of one activation tensor.
 *
 * Method: MegDet, section 3.3 "Cross-GPU Batch Normalization", Algorithm 1.
 *   steps 1-3   device sums            s[k,c] = sum over shard k of x
 *   steps 4-5   reduce + broadcast     mean[c] = (sum_k s[k,c]) / M
 *   steps 6-8   device variance sums   v[k,c] = sum over shard k of (x - mean[c])^2
 *   steps 9-10  reduce + broadcast     var[c]  = (sum_k v[k,c]) / M   (biased)
 *   step 11     y = gamma (x - mean)/sqrt(var + eps) + beta
 * with M = N*H*W the pooled count per channel.  The paper gives no backward;
 * the one here is the chain rule through the pooled mean and variance:
 *   a[k,c] = sum over shard k of dy,   b[k,c] = sum over shard k of dy*xhat
 *   dbeta = sum_k a,  dgamma = sum_k b,  xhat = (x - mean) * invstd
 *   dx = gamma * invstd * (dy - dbeta/M - xhat * dgamma/M)
 *
 * Conventions common to every entry point
 *   - Every tensor/vector pointer is a DEVICE pointer owned by the caller; the
 *     library never allocates, frees or keeps device memory.  Scratch is the
 *     caller's `workspace` (size from cgbn_workspace_bytes, contents undefined
 *     after a call).  Activation tensors (x, y, dy, dx) are dense in `layout`
 *     with element type `dtype`, their base address 16-byte aligned.  Per-channel
 *     vectors are float[C]; shard partials are double[K*C], index k*C + c.
 *   - Shard k holds images [k*N/K, (k+1)*N/K); 1 <= K <= N and N % K == 0.
 *   - All work is enqueued on `stream` (a hipStream_t passed as void*; NULL is
 *     the default stream).  No call synchronises, reads back or allocates, and scratch is
 *     cleared by kernels, so a sequence of calls can be captured into a HIP graph and
 *     replayed (with the same pointers).
 *   - Errors: the return code only.  Argument errors are found on the host
 *     before any launch and leave every output untouched.  CGBN_ERR_HIP wraps a
 *     failed launch.  NaN/Inf in the data are not errors; they propagate within
 *     their channel.  Per-row partial sums are floats (cross-row sums doubles), so
 *     a channel's squared deviations must stay inside float range (|x - mean| up
 *     to about 1e18) for the stated accuracy.
 *   - Aliasing: y may be exactly x, dx may be exactly dy; any other overlap of
 *     an output with another argument is undefined.
 *   - `mean_lo` (optional, may be NULL everywhere): float[C] holding the part of
 *     the pooled mean that does not fit `mean`'s float, mean + mean_lo being the
 *     mean to about double precision.  The forward uses it internally in any
 *     case; exporting it lets the backward see the same mean when |mean| is
 *     orders of magnitude above the channel's spread.
 *   - Concurrency: calls on ONE stream, or on several streams as long as they do not run at
 *     the same time, need nothing special.  cgbn_forward / cgbn_backward calls that may
 *     overlap in time on one device (different streams, each with its own workspace) must
 *     set the "cooperative" knob first: their single-launch kernels wait for sibling
 *     workgroups, and two such grids dispatched together could each end up half resident and
 *     starve the other until the bounded waits give up (error word set, NaN statistics).
 *     (Calls that take the column-slab or the flat kernels are exempt: no wait of the former needs its
 *     siblings resident and the latter have none, see "last_forward_slab" and "last_forward_flat" for
 *     which calls those are.)
 *     A workspace must never be shared by calls that can overlap.
 *   - Results are bitwise reproducible run to run (fixed summation order, no
 *     floating-point atomics) and depend on K only through rounding.
 */
#ifndef CGBN_H
#define CGBN_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Status, layout and dtype travel as plain ints (any value a caller passes is representable; values outside
 * the lists below are answered with CGBN_ERR_ENUM, or "unknown status"). */
typedef int cgbn_status;
enum {
    CGBN_OK = 0,
    CGBN_ERR_NULL = 1,       /* a required pointer is NULL */
    CGBN_ERR_SHAPE = 2,      /* a dimension is < 1 or the tensor is too large to index */
    CGBN_ERR_SHARD = 3,      /* K < 1, K > N or N % K != 0 */
    CGBN_ERR_ENUM = 4,       /* layout or dtype out of range */
    CGBN_ERR_EPS = 5,        /* eps is not finite and > 0 */
    CGBN_ERR_WORKSPACE = 6,  /* workspace NULL, misaligned (256 B) or too small */
    CGBN_ERR_ALIGN = 7,      /* an activation tensor is not 16-byte aligned */
    CGBN_ERR_HIP = 8,        /* the HIP runtime refused a launch */
    CGBN_ERR_TUNING = 9,     /* unknown tuning key or value out of range */
    CGBN_ERR_MOMENTUM = 10,  /* momentum outside [0, 1] */
    CGBN_ERR_ALIAS = 11,     /* two outputs that must differ are the same buffer */
    CGBN_ERR_SCRATCH = 12,   /* cgbn_forward_static: the problem needs more than CGBN_STATIC_SCRATCH_BYTES */
    CGBN_ERR_ACTIVATION = 13, /* an activation, rotation or scaling that is not in its list */
    CGBN_ERR_STRIDE = 14     /* rows of a strided tensor overlap */
};

typedef int cgbn_layout;
enum { CGBN_NCHW = 0, CGBN_NHWC = 1 };
typedef int cgbn_dtype;      /* of x, y, dy, dx */
enum { CGBN_F32 = 0, CGBN_BF16 = 1 };

/* Bytes of workspace any entry point below needs for this problem (a multiple
 * of 256; the workspace itself must be 256-byte aligned).  Returns 0 if the
 * arguments are invalid.  Host-only, launches nothing. */
size_t cgbn_workspace_bytes(int N, int C, int H, int W, cgbn_layout layout,
                            cgbn_dtype dtype, int K);

/* Byte offset, inside a workspace, of a 32-bit word that is 0 after cgbn_forward /
 * cgbn_backward unless a bounded device-side wait gave up (it cannot when the launch is
 * sound; if it does, the statistics of the affected channels are NaN).  The offset is the
 * same for every problem; (size_t)-1 if the arguments are invalid.  Callers that do not
 * want to read workspace memory themselves use cgbn_workspace_status. */
size_t cgbn_workspace_error_offset(int N, int C, int H, int W, cgbn_layout layout,
                                   cgbn_dtype dtype, int K);

/* The first-class way to learn of such a give-up: enqueues on `stream` a one-thread kernel
 * that sets *gave_up (a DEVICE int owned by the caller) to 1 if the error word of
 * `workspace` is up, and leaves it untouched otherwise.  Call it after the cgbn_forward /
 * cgbn_backward (or their ReLU variants) it is to watch, on the same stream and before the
 * next call that uses the workspace (every such call clears the word when it starts).  Zero
 * *gave_up once, let any number of layers raise it, and read it when the host next
 * synchronises anyway (once per training step, say): a non-zero value means that some
 * statistics of that step are NaN because the device was shared with other kernels in a way
 * the launch could not cope with (see "Concurrency" above and the "cooperative" knob). */
cgbn_status cgbn_workspace_status(const void* workspace, int* gave_up, void* stream);

/* Algorithm 1, all steps.  In: x, gamma[C], beta[C], eps.  Out: y (same shape,
 * layout and dtype as x; bf16 rounded to nearest-even), mean[C], invstd[C] =
 * 1/sqrt(var + eps), and mean_lo[C] if not NULL. */
cgbn_status cgbn_forward(const void* x, int N, int C, int H, int W, cgbn_layout layout, int K,
                         const float* gamma, const float* beta, float eps,
                         void* y, float* mean, float* invstd,
                         cgbn_dtype dtype, float* mean_lo,
                         void* workspace, size_t workspace_bytes, void* stream);

/* cgbn_forward for callers that can neither allocate device memory nor bring a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments,
 * kernels and results as cgbn_forward, without `workspace` / `workspace_bytes`: the scratch is a
 * static device array of CGBN_STATIC_SCRATCH_BYTES inside the library (each GPU the library runs
 * on holds one until the process ends).  The call allocates and frees nothing, on the device or
 * through any allocating library routine.
 *   - A problem whose cgbn_workspace_bytes exceeds CGBN_STATIC_SCRATCH_BYTES is refused with
 *     CGBN_ERR_SCRATCH before anything is launched (the five detector-shaped workloads of this
 *     repository need 0.01 to 8.1 MiB).
 *   - The array's device address is looked up on the first call on each device; make that call
 *     outside a graph capture.
 *   - Every call on a GPU uses that GPU's one array: calls that can overlap in time on one GPU
 *     (different streams) race on it and must not be made; back-to-back calls on one stream are
 *     fine (whatever must start cleared is cleared by kernels of the call itself).
 *   - The give-up word of the single-launch kernels lives in the array too; there is no
 *     workspace pointer to pass to cgbn_workspace_status, so watch it through NaN statistics. */
#define CGBN_STATIC_SCRATCH_BYTES (16u << 20)
cgbn_status cgbn_forward_static(const void* x, int N, int C, int H, int W, cgbn_layout layout, int K,
                                const float* gamma, const float* beta, float eps,
                                void* y, float* mean, float* invstd,
                                cgbn_dtype dtype, float* mean_lo, void* stream);

/* Backward of Algorithm 1's last step through the pooled statistics.  In: dy, x,
 * mean[C], invstd[C] as written by cgbn_forward, gamma[C], mean_lo[C] or NULL.
 * Out: dx, dgamma[C], dbeta[C]. */
cgbn_status cgbn_backward(const void* dy, const void* x, const float* mean, const float* invstd,
                          const float* gamma, void* dx, float* dgamma, float* dbeta,
                          int N, int C, int H, int W, cgbn_layout layout, int K,
                          cgbn_dtype dtype, const float* mean_lo,
                          void* workspace, size_t workspace_bytes, void* stream);

/* ---- CGBN followed by a shortcut add and a ReLU, the two placements of a normalization
 * layer in the detector's backbone (ResNet-50, section 4): y = max(0, z) inside a block,
 * y = max(0, z + shortcut) at a block's end, z being Algorithm 1's output.  The paper does
 * not discuss the activation; fusing it here saves the separate sweeps over y and dy. ---- */

/* As cgbn_forward, then y = max(0, z + shortcut).  `shortcut` (same shape, layout and
 * dtype as x) may be NULL: y = max(0, z).  The statistics are those of x alone.
 * y may be exactly x or exactly shortcut. */
cgbn_status cgbn_forward_relu(const void* x, const void* shortcut, int N, int C, int H, int W,
                              cgbn_layout layout, int K, const float* gamma, const float* beta, float eps,
                              void* y, float* mean, float* invstd, cgbn_dtype dtype, float* mean_lo,
                              void* workspace, size_t workspace_bytes, void* stream);

/* Its backward.  `y` is the output cgbn_forward_relu stored: gradient passes where y > 0
 * (dz = dy there, 0 elsewhere), then dbeta, dgamma, dx as in cgbn_backward with dz for dy.
 * `dshortcut`, if not NULL, receives dz (the gradient of the shortcut).  dx may be exactly
 * dy, or dshortcut may be exactly dy; dx and dshortcut must differ (CGBN_ERR_ALIAS). */
cgbn_status cgbn_backward_relu(const void* dy, const void* y, const void* x,
                               const float* mean, const float* invstd, const float* gamma,
                               void* dx, void* dshortcut, float* dgamma, float* dbeta,
                               int N, int C, int H, int W, cgbn_layout layout, int K,
                               cgbn_dtype dtype, const float* mean_lo,
                               void* workspace, size_t workspace_bytes, void* stream);

/* ---- The same path one step at a time, one sweep over the tensor per call.
 * cgbn_forward and cgbn_backward run these kernels back to back where a shape
 * qualifies neither for the single-launch NCHW kernels nor for the column-slab kernels (and always when the
 * "fused" knob is 0).  Meant for tests and measurement. ---- */

/* Algorithm 1 steps 1-3: s[k*C + c] = sum over shard k of x. */
cgbn_status cgbn_shard_sum(const void* x, int N, int C, int H, int W, cgbn_layout layout, int K,
                           cgbn_dtype dtype, double* s,
                           void* workspace, size_t workspace_bytes, void* stream);

/* Steps 4-5: mean[c] = (sum_k s[k,c]) / M, with M given as a count.  mean_lo optional. */
cgbn_status cgbn_reduce_mean(const double* s, int K, int C, long long M,
                             float* mean, float* mean_lo, void* stream);

/* Steps 6-8: v[k*C + c] = sum over shard k of (x - mean[c])^2 (mean_lo optional). */
cgbn_status cgbn_shard_sqdev(const void* x, int N, int C, int H, int W, cgbn_layout layout, int K,
                             cgbn_dtype dtype, const float* mean, const float* mean_lo, double* v,
                             void* workspace, size_t workspace_bytes, void* stream);

/* Steps 9-10: invstd[c] = 1/sqrt((sum_k v[k,c])/M + eps). */
cgbn_status cgbn_reduce_invstd(const double* v, int K, int C, long long M, float eps,
                               float* invstd, void* stream);

/* Step 11: y = gamma*(x - mean)*invstd + beta. */
cgbn_status cgbn_normalize(const void* x, int N, int C, int H, int W, cgbn_layout layout,
                           cgbn_dtype dtype, const float* mean, const float* mean_lo,
                           const float* invstd, const float* gamma, const float* beta,
                           void* y, void* stream);

/* Backward device sums: a[k*C + c] = sum dy, b[k*C + c] = sum dy*xhat over shard k. */
cgbn_status cgbn_backward_shard_sums(const void* dy, const void* x, int N, int C, int H, int W,
                                     cgbn_layout layout, int K, cgbn_dtype dtype,
                                     const float* mean, const float* mean_lo, const float* invstd,
                                     double* a, double* b,
                                     void* workspace, size_t workspace_bytes, void* stream);

/* Backward reduce: dbeta[c] = sum_k a[k,c], dgamma[c] = sum_k b[k,c]. */
cgbn_status cgbn_backward_reduce(const double* a, const double* b, int K, int C,
                                 float* dbeta, float* dgamma, void* stream);

/* dx = gamma*invstd*(dy - dbeta/M - xhat*dgamma/M). */
cgbn_status cgbn_backward_dx(const void* dy, const void* x, int N, int C, int H, int W,
                             cgbn_layout layout, cgbn_dtype dtype,
                             const float* mean, const float* mean_lo, const float* invstd,
                             const float* gamma, const float* dgamma, const float* dbeta,
                             void* dx, void* stream);

/* ---- Fixed-statistics ("frozen") mode: the layer the paper's baseline detectors use
 * (section 3.1; opening of section 3.3; Table 3, row "16-base", BN size 0), where the
 * statistics are constants computed beforehand.  One elementwise sweep each; no
 * workspace.  The paper does not say how the constants come about; the update below is
 * the exponential moving average of the batch-normalization work section 3.3 builds on,
 * with `momentum` and `unbiased` left to the caller. ---- */

/* y = gamma*(x - fixed_mean)/sqrt(fixed_var + eps) + beta: the formula of Algorithm 1's last
 * step with constants for the statistics.  fixed_mean[C], fixed_var[C] (variances, not
 * their inverse roots), gamma[C], beta[C].  y may be exactly x. */
cgbn_status cgbn_frozen_forward(const void* x, int N, int C, int H, int W, cgbn_layout layout,
                                cgbn_dtype dtype, const float* fixed_mean, const float* fixed_var,
                                const float* gamma, const float* beta, float eps,
                                void* y, void* stream);

/* Its backward.  Statistics and affine parameters are constants of the layer, so
 * dx = dy*gamma/sqrt(fixed_var + eps) and there is no dgamma/dbeta.  dx may be exactly dy. */
cgbn_status cgbn_frozen_backward(const void* dy, int N, int C, int H, int W, cgbn_layout layout,
                                 cgbn_dtype dtype, const float* fixed_var, const float* gamma,
                                 float eps, void* dx, void* stream);

/* After a cgbn_forward with the same eps over M = N*H*W values per channel:
 *   running_mean <- (1-momentum)*running_mean + momentum*(mean + mean_lo)
 *   running_var  <- (1-momentum)*running_var  + momentum*var*(unbiased ? M/(M-1) : 1)
 * in place, with var = 1/invstd^2 - eps (accurate to about 2e-7*(var + eps)).  mean_lo may
 * be NULL.  0 <= momentum <= 1, else CGBN_ERR_MOMENTUM; unbiased needs M >= 2. */
cgbn_status cgbn_update_running_stats(const float* mean, const float* mean_lo, const float* invstd,
                                      float eps, long long M, int C, float momentum, int unbiased,
                                      float* running_mean, float* running_var, void* stream);

/* ---- The layers beside the normalization: matrix product with bias, residual and activation; the gated feed-forward
 * block; the per-head norm of queries and keys with the rotation by position.  Rows are tokens, pixels or crops: a
 * channels-last map [N][H][W][C] is M = N*H*W rows of C values, and a 1x1 convolution of it is cgbn_linear_forward
 * (a fixed-statistics layer folds into its weights and bias, the shortcut and the ReLU are its residual and activation).
 *   - Tensors are dense row by row (but for the strides of cgbn_head_norm_*), their element type `dtype` (weights too), base
 *     addresses 16-byte aligned; widths may be odd.  Bias vectors, norm weights and their gradients are float.
 *   - Sums are held in 32 bits and results rounded once, to nearest even; what a backward pass hands from one of its kernels
 *     to the next (dz, dg, du below) is rounded to `dtype`.  Float products are formed from three bfloat16 parts a value, which are
 *     exact, and are off by less than 2^-22 of themselves (values under 1e-33 have fewer bits); with few rows by float instructions.
 *   - M (or T) may be 0: forward calls do nothing, backward calls write zero weight gradients.
 *   - Outputs and inputs are different buffers unless said otherwise (equal pointers where that is wrong are answered with
 *     CGBN_ERR_ALIAS; partial overlaps are undefined).  The workspace may be NULL where the size below is not more than 256.
 *   - Nothing waits for a sibling workgroup: calls on different streams may overlap, each with its own workspace.
 *   - NaN and infinities are not errors; they reach the results whose sums they enter, and no others. ---- */

/* Of z: z; max(0, z); z * Phi(z) with the normal distribution's Phi; z / (1 + exp(-z)).  For float tensors Phi of negative z and the exponential are
 * within 16 and 8 units of 2^-24 of themselves; for bfloat16 ones Phi is within 2.7e-7.  Of -infinity the last two, and of infinities their slopes, are NaN. */
typedef int cgbn_activation;
enum { CGBN_ACT_NONE = 0, CGBN_ACT_RELU = 1, CGBN_ACT_GELU = 2, CGBN_ACT_SILU = 3 };

/* Bytes of workspace for M rows of K values in, N out (backward: 0 or 1).  0 if the arguments are invalid. */
size_t cgbn_linear_workspace_bytes(long long M, int N, int K, cgbn_dtype dtype, int backward);

/* z = x w^T + bias + residual, y = act(z).  In: x[M][K], w[N][K], bias[N] or NULL, residual[M][N] or NULL.  Out: y[M][N],
 * and z[M][N] if not NULL (what the backward of GELU and SiLU starts from).  y may be exactly residual. */
cgbn_status cgbn_linear_forward(const void* x, const void* w, const float* bias, const void* residual, long long M, int N,
                                int K, cgbn_activation act, void* y, void* z, cgbn_dtype dtype,
                                void* workspace, size_t workspace_bytes, void* stream);

/* Its backward: dz = dy * act'(z), dx = dz w, dw = dz^T x, dbias = sum over rows of dz, dresidual = dz.  `saved` is the
 * stored y for ReLU (gradient passes where y > 0), the stored z for GELU and SiLU, and not read without an activation.
 * Outputs may be NULL where they are not wanted.  dresidual may be exactly dy. */
cgbn_status cgbn_linear_backward(const void* dy, const void* x, const void* w, const void* saved, long long M, int N, int K,
                                 cgbn_activation act, void* dx, void* dw, float* dbias, void* dresidual, cgbn_dtype dtype,
                                 void* workspace, size_t workspace_bytes, void* stream);

size_t cgbn_gated_workspace_bytes(long long M, int F, int K, cgbn_dtype dtype, int backward);

/* g = x w_gate^T, u = x w_up^T, h = act(g) * u, one kernel.  In: x[M][K], w_gate[F][K], w_up[F][K].  Out: h[M][F], and
 * gate[M][F] = g, up[M][F] = u if not NULL (both or neither), which the backward starts from. */
cgbn_status cgbn_gated_forward(const void* x, const void* w_gate, const void* w_up, long long M, int F, int K,
                               cgbn_activation act, void* h, void* gate, void* up, cgbn_dtype dtype,
                               void* workspace, size_t workspace_bytes, void* stream);

/* Its backward: dg = dh * u * act'(g), du = dh * act(g), dx = dg w_gate + du w_up, dw_gate = dg^T x, dw_up = du^T x.
 * dx may be NULL, and so may dw_gate and dw_up (both or neither). */
cgbn_status cgbn_gated_backward(const void* dh, const void* x, const void* w_gate, const void* w_up, const void* gate,
                                const void* up, long long M, int F, int K, cgbn_activation act, void* dx, void* dw_gate,
                                void* dw_up, cgbn_dtype dtype, void* workspace, size_t workspace_bytes, void* stream);

/* Which values of a head are turned together: i and i + R/2, or 2i and 2i + 1, for i in [0, R/2). */
typedef int cgbn_rotation;
enum { CGBN_ROTATE_HALVES = 0, CGBN_ROTATE_PAIRS = 1 };

/* Every row x[D] (one head of one token): n = weight * x / sqrt(mean(x^2) + eps), then its first R values are rotated by the
 * token's position: (a, b) -> (a c - b s, b c + a s) with c = cos[p][i], s = sin[p][i], p = positions[token] (the token's
 * own index if positions is NULL).  R = 0: no rotation, positions, cos and sin are not read.
 *   q: Hq heads of D values side by side in each of T rows, row to row `ldq` elements (q and k may be slices of a joint
 *   projection's rows); k: Hk heads, `ldk`; Hk may be 0, k, wk and yk are then not read.  wq[D], wk[D]; cos, sin
 *   [table_rows][R/2]; outputs with strides of their own; yq may be exactly q (with its stride), yk exactly k.
 *   1 <= D <= 1024, R even.  A position outside [0, table_rows) reads nothing and makes the R rotated values of its rows NaN. */
cgbn_status cgbn_head_norm_forward(const void* q, long long ldq, const void* k, long long ldk, long long T, int Hq, int Hk,
                                   int D, int R, cgbn_rotation style, const int* positions, const float* cos,
                                   const float* sin, int table_rows, const float* wq, const float* wk, float eps,
                                   void* yq, long long ldyq, void* yk, long long ldyk, cgbn_dtype dtype, void* stream);

/* Bytes of workspace of its backward. */
size_t cgbn_head_norm_workspace_bytes(long long T, int Hq, int Hk, int D, cgbn_dtype dtype);

/* Its backward, from the layer's inputs q and k: dq, dk, and the weights' gradients dwq[D], dwk[D] summed over all tokens and
 * heads.  dq may be exactly dyq (with its stride), dk exactly dyk.  A position outside the table makes its rows' gradients
 * NaN, and with them dwq and dwk. */
cgbn_status cgbn_head_norm_backward(const void* dyq, long long lddyq, const void* dyk, long long lddyk, const void* q,
                                    long long ldq, const void* k, long long ldk, long long T, int Hq, int Hk, int D, int R,
                                    cgbn_rotation style, const int* positions, const float* cos, const float* sin,
                                    int table_rows, const float* wq, const float* wk, float eps, void* dq, long long lddq,
                                    void* dk, long long lddk, float* dwq, float* dwk, cgbn_dtype dtype,
                                    void* workspace, size_t workspace_bytes, void* stream);

/* ---- Serving: rotation by position without a norm, a cache of keys and values in pages, attention over it.  The conventions of the layers
 * above hold (types, alignment, sums in 32 bits, statuses, streams; calls on different streams may overlap, each with its own workspace).
 * The cache of one layer is two pools of `pages` pages, k_pages and v_pages[pages][Hk][page][D]: a page holds `page` tokens (a power of two up to 1024),
 * head by head.  A request's tokens lie in the pages that its row of `table` names, in order; the prefix that all requests of a
 * batch share lies in the pages of a table of its own, is `prefix` tokens long and precedes the first token of each.  A place (slot) in the pools is page id * page + token
 * in page; pages * page < 2^31.  Page ids outside [0, pages) are no error: they stand for pages that are not there. ---- */

/* How the frequencies of a rotation are stretched for contexts longer than those a model was trained on, by `factor` >= 1 (f[i] = base^(-2i / R)):
 * f / factor; with base * factor^(R / (R - 2)) for the base; by parts, g f + (1 - g) f / factor with g = (turns - slow) / (fast - slow)
 * within [0, 1] and turns = trained f / (2 pi), the turns that a pair made over the `trained` positions. */
typedef int cgbn_scaling;
enum { CGBN_SCALE_NONE = 0, CGBN_SCALE_POSITIONS = 1, CGBN_SCALE_BASE = 2, CGBN_SCALE_PARTS = 3 };

/* The R/2 frequencies, radians a position, to HOST memory.  Host-only, launches nothing.  base > 1; trained, fast and slow (trained >= 1,
 * fast > slow >= 0) are looked at by parts alone. */
cgbn_status cgbn_rotary_frequencies(int R, double base, cgbn_scaling scaling, double factor, double trained, double fast, double slow,
                                    double* freq);

/* The first R values of every head of D are turned by the token's position (a, b) -> magnitude (a cos t - b sin t, b cos t + a sin t) with t = p freq[i],
 * p = positions[token] (any int; the token's own index if positions is NULL), freq[R/2] a DEVICE vector of doubles; the others are copied.  Rows, heads, strides and
 * `style` as in cgbn_head_norm_forward; Hk may be 0; yq may be exactly q (with its stride), yk exactly k.  Turns are counted in 64 bits: an angle is off by
 * less than 1.3 * 2^-52 of itself (2^-20 radians at position 2^31 of the fastest pair), its cosine and sine by 2^-23 beside that.  Up to 2^14 heads, T <= 2^30, T (Hq + Hk) <= 2^33. */
cgbn_status cgbn_rotate_forward(const void* q, long long ldq, const void* k, long long ldk, long long T, int Hq, int Hk, int D, int R,
                                cgbn_rotation style, const int* positions, const double* freq, float magnitude, void* yq, long long ldyq,
                                void* yk, long long ldyk, cgbn_dtype dtype, void* stream);

/* Its backward: gradients turned back, times magnitude.  dq may be exactly dyq (with its stride), dk exactly dyk. */
cgbn_status cgbn_rotate_backward(const void* dyq, long long lddyq, const void* dyk, long long lddyk, long long T, int Hq, int Hk, int D, int R,
                                 cgbn_rotation style, const int* positions, const double* freq, float magnitude, void* dq, long long lddq,
                                 void* dk, long long lddk, cgbn_dtype dtype, void* stream);

/* Bytes of workspace of a plan. */
size_t cgbn_page_plan_workspace_bytes(int B, long long T);

/* The plan of a step: request b has have[b] tokens of its own in the cache and gets fresh[b] (either may be 0; less counts as 0).  All of it on the device.
 *   rows[B + 1]     where each request's new tokens start among the step's T rows, in order; tokens beyond row T are cut off
 *   lengths[B]      tokens of its own after the step
 *   table[B][max_pages]  in and out: pages that a request needs beyond those that have[b] tokens take come from free_pages[free_count], in order,
 *                   from the taken[0]-th on, first request first; where the list or the row of the table is at its end there are none (-1 in the table)
 *   slots[T], positions[T]   each row's place in the cache (-1: it has none) and its position, `before` (the prefix's length) + its index
 *                   in its request; rows behind the last token: -1 and 0
 *   counts[2]       pages of the list that are taken now; new tokens that got no place (slot -1, also in a page that is not there, of the list or of
 *                   the table, as behind the end of the list in later steps) or no row (at most 2^31 - 1).  counts may be exactly taken.
 * have[b] is cut to max_pages * page.  0 <= before <= 2^30, B <= 2^20, T <= 2^29, 1 <= max_pages <= 2^16, free_count < 2^30. */
cgbn_status cgbn_page_plan(const int* have, const int* fresh, int B, int before, const int* free_pages, int free_count, const int* taken,
                           int* counts, int* table, int max_pages, int pages, int page, long long T, int* rows, int* lengths, int* slots,
                           int* positions, void* workspace, size_t workspace_bytes, void* stream);

/* Puts T tokens' keys and values (Hk heads of D values side by side, row to row ldk and ldv elements, rows on 16 bytes) to their places in
 * the pages; tokens whose slot is outside the pools are left out.  Two tokens of one call have different slots (of equal ones either may stay, in parts).
 * D a multiple of 8 up to 256, Hk <= 1024, T <= 2^30. */
cgbn_status cgbn_page_store(const void* k, long long ldk, const void* v, long long ldv, long long T, int Hk, int D, const int* slots,
                            void* k_pages, void* v_pages, int pages, int page, cgbn_dtype dtype, void* stream);

/* Bytes of workspace of the attention below; capacity: max_pages * page. */
size_t cgbn_prefix_attention_workspace_bytes(long long T, int B, int Hq, int Hk, int D, long long prefix, long long capacity,
                                             cgbn_dtype dtype);

/* out = softmax(scale q k^T) v, head by head, of the T rows' queries (Hq heads of D values, Hq a multiple of Hk: head h reads keys of head h / (Hq / Hk)).
 * Request b's queries are rows rows[b] ... rows[b + 1] - 1 (rows[0] = 0, ascending), its last tokens: the j-th of n sees the prefix and its request's tokens up to
 * itself, the first lengths[b] - n + j + 1.  rows may be NULL: one row each, T = B.  Rows behind rows[B] are left as they were.
 * A row that sees no key is zero.  lse[T][Hq], if not NULL: the logarithm of the sum of the exponentials of a row's scores, -infinity where there is no key.
 *   Keys beyond lengths[b], in pages that are not there, or later than a row's own are not looked at, whatever their places hold. lengths[b] may be more than
 *   max_pages * page, as a plan's are: tokens that the table has no room for are not there, and count where a row's own token is.  max_pages = 0: no own tokens,
 *   table and lengths are not read.  Weights are rounded to bfloat16 for the products of bfloat16 tensors, their sum is not.
 * Weights times values are summed before they are divided: values above about 1e33 over the number of keys may overflow.
 * A row whose scores are all -infinity (of infinite queries or keys) is zero, as one without keys.
 *   D a multiple of 8 up to 256; Hq <= 1024; rows of q and out on 16 bytes; T * Hq < 2^26 - 3, B <= 2^20, B * Hk <= 2^22; max_pages <= 2^20, prefix and
 *   max_pages * page < 2^30. */
cgbn_status cgbn_prefix_attention(const void* q, long long ldq, long long T, int B, const int* rows, const int* lengths, int Hq, int Hk,
                                  int D, float scale, const void* k_pages, const void* v_pages, int pages, int page,
                                  const int* prefix_table, int prefix, const int* table, int max_pages, void* out, long long ldo,
                                  float* lse, cgbn_dtype dtype, void* workspace, size_t workspace_bytes, void* stream);

/* ---- housekeeping ---- */

/* Static, never NULL. */
const char* cgbn_status_string(cgbn_status status);

/* Launch-shape knobs for measurement sweeps.  They are process-wide; reading and writing
 * them is serialised, and every call of the library works on ONE copy of them, taken when it
 * starts (or when its thread made the plan for an earlier call, if no knob has changed
 * since), so calls from several host threads are safe and a call never sees half of a
 * change.  The workspace size depends on some of them: re-query cgbn_workspace_bytes after
 * a change (a call whose workspace is too small for the knobs it runs under returns
 * CGBN_ERR_WORKSPACE before launching anything).
 *   "chunk_bytes"      NCHW: bytes of one plane handled by one workgroup
 *   "wave_plane_bytes" NCHW: planes up to this size are handled by one wavefront
 *   "flat"             0/1 (default 1): NCHW channels that fit one workgroup's registers (up to 64 KiB; 128 KiB where
 *                      channels are few) go through the flat kernels, one launch with nothing handed over
 *   "tiny_planes"      0/1 (default 1): NCHW planes of at most 2 KiB, C a multiple of 8: a workgroup of the
 *                      multi-sweep kernels takes a run of 8 ... 256 planes of consecutive channels at once
 *   "piece_bytes"      NHWC reductions: bytes of one pixel range handled by one workgroup (0, the default:
 *                      chosen per shape so that the grid fills the device's compute units evenly)
 *   "map_piece_bytes"  NHWC normalise / dx: the same for the elementwise sweeps (0, the default: 32 KiB, 16 for three
 *                      float tensors; shorter for small tensors, and where C is no whole number of vectors and
 *                      pixels cannot be grouped; longer for rows of several tiles)
 *   "reverse"          0/1: alternate the sweep direction between consecutive sweeps
 *   "nt_store"         0/1: non-temporal stores for y and dx
 *   "fused"            0/1: register-resident forward/backward in one launch (the NCHW kernels and the
 *                      column-slab kernels; 0: separate sweeps)
 *   "one_sweep_stats"  0/1 (default 1): where cgbn_forward runs as separate sweeps, steps 1-10 come from ONE sweep
 *                      over x: each row partial is the sum about a per-channel pivot and M2, the squared
 *                      deviations from the row's own mean (formed chunk by chunk in registers, never as a
 *                      difference of large sums); the combine step turns them into Algorithm 1's sums about the
 *                      pooled mean by the pairwise update.  3 tensor sweeps instead of 4, same results up to
 *                      rounding.  0: one sweep for the sums, a second for the squared deviations (what the
 *                      step-by-step entry points below always do); channels-last forwards then run as
 *                      separate sweeps whatever their shape
 *   "cooperative"      0/1 (default 0): launch the single-launch kernels cooperatively, so that the runtime
 *                      guarantees the whole grid is resident; needed only if such calls can overlap on
 *                      different streams; costs about 15 us per launch
 *   "big_lds"          0/1 (default 1): NCHW shapes with at most 384 rows and 48 (large planes) or 128 (small
 *                      planes) shards use variants of the single-launch kernels that stage few rows and keep
 *                      more unit data in LDS
 *   "fused_groups"     workgroups of that launch (0 = all that are resident at once)
 *   "stagger"          0/1 (default 1): the single-launch kernels start their channel slots class by class, so
 *                      that the slots' load, hand-over and write-out phases interleave
 *   "stagger_us"       microseconds by which the last class starts after the first (0, the default: chosen
 *                      per launch, none for short launches)
 *   "stagger_phases"   number of such classes (2..64, default 16)
 *   "spin_limit"       polls before a device-side wait gives up (0: at once; for tests of that path)
 *   "wait_us"          microseconds of wall-clock time before it gives up (default 100000); once one wait
 *                      of a launch has given up, its later waits do so at once
 * The column-slab kernels take "fused", "one_sweep_stats", "nt_store", "fused_groups" (never fewer than a slab's units) and
 * "spin_limit"; there a unit that waits longer (or 300 us, 30 us once some unit has) gives nothing up, it moves
 * on and is finished by another.  "cooperative", "big_lds", "stagger", "stagger_us", "stagger_phases" and "wait_us" do not
 * concern them; their own backstop, for waits that end within microseconds in a sound launch, is a second.
 * cgbn_get_tuning returns -1 for an unknown key. */
cgbn_status cgbn_set_tuning(const char* key, long long value);
/* also readable: "last_forward_fused", "last_backward_fused" (1 if the last
 * cgbn_forward / cgbn_backward took the single-launch NCHW kernels), "last_forward_slab",
 * "last_backward_slab" (1 if it took the column-slab kernels), "last_forward_slab_vector",
 * "last_backward_slab_vector" (the bytes of their vectors, 16 or 8, or 0), "plans_made" (launch plans the calling thread has
 * made: calls come back to the last ones it keeps), "last_forward_flat", "last_backward_flat" (1 if it took the flat
 * kernels), "last_forward_edge", "last_backward_edge" (1 if it took those for planes that are no multiple of 16 bytes); "last_forward_fused" is 1 in
 * either case */
long long cgbn_get_tuning(const char* key);

/* One number of the launch plan the library would use for this problem under the current
 * knobs; host-only, launches nothing, -1 for invalid arguments or an unknown key.  For tests
 * of the host-side planning (every kernel trusts these numbers for its indexing).
 * Multi-sweep kernels: "grid" (workgroups of a reduction sweep), "gridm" (of a channels-last
 * elementwise sweep), "rows" / "rps" (row partials per channel / per shard), "G" (lanes adding
 * one shard's rows), "part_bytes" / "shard_bytes" (workspace bytes of one array of row partials /
 * of shard sums); NCHW: "wave_mode" (one wavefront per plane), "L" / "sp" (chunk elements, chunks
 * per plane); NHWC: "vec" (elements per access), "cv" (accesses per pixel), "TW" / "ctiles"
 * (accesses per pixel handled by one workgroup, workgroups per pixel), "rpp" (pixels per pass),
 * "PL" / "pps" (pixels per piece, pieces per shard; reductions), "PLm" / "ppsm" / "gridm" (elementwise with one input;
 * with a 2 or 3 behind them: two, three inputs), "single_consts" (elementwise with two inputs: constants by single loads).
 * NHWC, C no multiple of a 16-byte vector ("vec" 1): "may_group" (pixels that are taken as one pixel of whole vectors
 * where that pays, 1: never), "group_sums" / "group_sums_dy" (reductions of x, of x and dy, that do), "group_map" /
 * "group_map2" (elementwise sweeps with one input, with more), and of the plan then used "grouped_K", "grouped_cv",
 * "grouped_ctiles", "grouped_rows", "grouped_spix" (groups per shard), "grouped_PL", "grouped_pps".
 * Single-launch kernels, prefix "fwd_" or "bwd_": "ok" (the shape qualifies), "LB" (bytes per
 * access), "LPPC" (register slots per small plane; 0: large planes), "LPP" (slots a plane fills),
 * "IPU" (images per unit), "U" (units per channel), "tp" / "TL" (tiles per large plane, tile
 * elements), "rows", "rps", "G", "big" (0, or which LDS variant), "total_units", "last_plane" (byte offset of a unit's last plane
 * from its first).  Prefix "efwd_" or "ebwd_": the same of the plan for planes that are no multiple of 16 bytes, and "taken", "taken2" (calls
 * take it; calls with a shortcut, masked ones).  Flat kernels: "flat_waves" (wavefronts per channel, 0: the shape does not qualify), "flat_LB" (bytes of a vector),
 * "flat_S" (vectors per lane), "flat_vecs", "flat_total" (of a plane, of a channel), "flat_fwd", "flat_fwds", "flat_bwd", "flat_bwdm" (calls take them: forward, with a
 * shortcut, backward, masked).
 * Column-slab kernels, prefix "sfwd_" or "sbwd_" ("sfwds_": the forward with a shortcut, "sbwdm_": the masked backward): "ok" (the shape takes them instead of
 * sweeps), "first" (... also before the single-launch NCHW kernels), "vecs" (16-byte vectors per row of
 * the matrix), "R" (its rows), "cpc" (columns per channel), "cols" (vectors per slab), "slabs", "nch" (channels per slab, rounded up to a power of two), "rpp" (rows per pass),
 * "tpc" (threads that add one channel's partial sums), "U" (units per slab), "rpu" (rows per unit),
 * "P" (vectors per thread of the kernel variant).  Prefix "nfwd_", "nbwd_", "nfwds_", "nbwdm_": the same of the plan with 8-byte
 * vectors that takes its place if its own "ok" is 1.  Prefix "xfwd_", "xbwd_", "xbwdm_": the same of the plan in several rounds of slabs that share lines, where
 * the others are not "ok". */
long long cgbn_plan_get(int N, int C, int H, int W, cgbn_layout layout, cgbn_dtype dtype, int K,
                        const char* key);

/* A plain device-to-device copy of `bytes` bytes (a multiple of 16, both
 * pointers 16-byte aligned) by a kernel of this library: it reads and writes a
 * known number of bytes, which is what hardware traffic counters are calibrated
 * against when the library's kernels are profiled. */
cgbn_status cgbn_calibration_copy(const void* src, void* dst, size_t bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CGBN_H */
