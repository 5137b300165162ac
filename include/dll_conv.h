/*
 * dll_conv.h — C ABI of the MI355X (gfx950) implementation of the batched
 * 2D-convolution hot path of DLL (arxiv 1804.04512).
 *
 * What the paper defines (Section II-A): every minibatch of N images is convolved with
 * K kernels; the forward pass uses a "valid" convolution (the map shrinks), the backward
 * pass a "full" convolution (the map expands back), a third convolution of the layer
 * input with the output gradient yields the filter gradient; dense layers are matrix
 * products; activations and gradient operations are fused around them; all arithmetic
 * is single precision and works on whole minibatches; kernels are launched
 * asynchronously and data stays on the device.
 *
 * Conventions shared by every entry point
 *   - Every data pointer is a DEVICE pointer to a contiguous, row-major tensor.  fp32
 *     unless stated; labels are int32; pooling indices are one byte each.
 *   - The CALLER owns all memory.  The library never allocates, frees or keeps a pointer
 *     after the call returns.  Scratch comes from `ws` (`ws_bytes` >= the matching
 *     *_workspace_bytes query, 256-byte aligned); its contents are undefined afterwards.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls
 *     enqueue work and return without synchronising.
 *   - Layouts: x [N][C][H][W]; w [K][C][R][S]; bias [K]; stride 1;
 *     Ho = H + 2*pad - R + 1, Wo = W + 2*pad - S + 1;
 *     y and pool_idx [N][K][Ho/pool][Wo/pool].
 *   - `dy` always means the gradient w.r.t. the layer OUTPUT y (after activation and
 *     pooling); the library applies the pooling/activation derivative itself.
 *   - Errors are reported as dll_status before anything is launched: a missing required
 *     pointer -> DLL_ERR_NULL; non-positive sizes, a filter larger than the padded input,
 *     pad > R-1 or S-1, pooling on an odd map, an input aliasing an output (exact pointer
 *     equality only; partial overlap is undetected and undefined) -> DLL_ERR_SHAPE; an
 *     activation or pooling mode outside the enums, or a tensor of 2^31 or more elements
 *     -> DLL_ERR_UNSUPPORTED; a workspace that is too small or misaligned ->
 *     DLL_ERR_WORKSPACE; a failed launch -> DLL_ERR_DEVICE.  No exception crosses the ABI.
 */
#ifndef DLL_CONV_H
#define DLL_CONV_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DLL_OK = 0,
  DLL_ERR_NULL = 1,
  DLL_ERR_SHAPE = 2,
  DLL_ERR_UNSUPPORTED = 3,
  DLL_ERR_WORKSPACE = 4,
  DLL_ERR_DEVICE = 5,
  DLL_ERR_SCRATCH_LIMIT = 6 /* dll_conv_valid_wgrad_noalloc only: the layer needs more than its built-in scratch */
} dll_status;

/* Activation functions the paper's networks use (Sections II-B, IV-B, V, VI). */
typedef enum { DLL_ACT_IDENTITY = 0, DLL_ACT_SIGMOID = 1, DLL_ACT_RELU = 2 } dll_act;

/* One stride-1 convolution layer (Section II-A: N images, K kernels). */
typedef struct {
  int N, C, H, W; /* input minibatch, NCHW                                        */
  int K, R, S;    /* K filters of C x R x S                                       */
  int pad;        /* zeros added on every side; 0 = the paper's "valid"           */
  int act;        /* dll_act applied to conv + bias                               */
  int pool;       /* 1 = none, 2 = 2x2 stride-2 max pooling (Ho and Wo even)      */
} dll_conv_desc;

/* One fully-connected layer, weights [out][in] (Section II-A). */
typedef struct {
  int in, out, act;
} dll_dense_desc;

/* A CNN: n_conv convolution layers (all with the same N, each consuming the previous
 * one's output), flattened NCHW row-major into n_dense dense layers; the last dense layer
 * is linear (its `act` is ignored) and feeds a softmax cross-entropy over `classes`.
 * n_conv may be 0: then the network is fully connected (Section IV-A), its input x is
 * [batch][dense[0].in] and `batch` gives the mini-batch size; with n_conv > 0 `batch` is
 * ignored (the batch is conv[0].N) and `conv` must not be NULL. */
typedef struct {
  int n_conv;
  const dll_conv_desc *conv; /* host pointer */
  int n_dense;
  const dll_dense_desc *dense; /* host pointer */
  int classes;
  int batch;
} dll_net_desc;

/* Visible unit types of the RBM steps (Section II). */
typedef enum { DLL_VISIBLE_BINARY = 0, DLL_VISIBLE_GAUSSIAN = 1 } dll_visible_unit;

const char *dll_status_string(dll_status s);

/* Bytes of scratch the three single-layer calls below need at most (host computation). */
size_t dll_conv_workspace_bytes(const dll_conv_desc *d);

/* Forward layer (Section II-A: the valid convolution of the forward pass):
 *   z[n,k,i,j] = bias[k] + sum_{c,r,s} xpad[n,c,i+r,j+s] * w[k,c,r,s]
 *   y = maxpool2x2(act(z)) when pool == 2, else act(z)
 * pool_idx (required iff pool == 2) receives, in bits 0-1 of each byte, 2*a+b of the window's
 * maximum (first one in the order (0,0),(0,1),(1,0),(1,1) on ties of the pre-activation).
 * When act is ReLU, bit 2 (value 4) is also set where the pooled output is zero, i.e. where
 * the unit passes no gradient; all other bits are zero.  bias may be NULL. */
dll_status dll_conv_valid_fwd(const dll_conv_desc *d, const float *x, const float *w,
                              const float *bias, float *y, unsigned char *pool_idx, void *ws,
                              size_t ws_bytes, void *stream);

/* Backward-data layer (Section II-A: the full convolution of the backward pass):
 *   dz = unpool(dy, pool_idx) * act'(y)          (never stored)
 *   dx[n,c,i,j] = sum_{k,r,s} dz[n,k,i+pad-r,j+pad-s] * w[k,c,r,s]
 * pool_idx is required iff pool == 2; only bits 0-1 of its bytes are read when y is given.
 * y may be NULL when act is the identity.  y may also be NULL when act is ReLU and pool == 2:
 * then act'(y) is taken from bit 2 of pool_idx as dll_conv_valid_fwd wrote it (zero gradient
 * where the bit is set) and the layer output is not read at all. */
dll_status dll_conv_full_bwd(const dll_conv_desc *d, const float *dy, const float *y,
                             const unsigned char *pool_idx, const float *w, float *dx, void *ws,
                             size_t ws_bytes, void *stream);

/* The same backward-data layer computed through the Fourier transform (Section II-A's first
 * implementation of the full convolution: image and filter padded to the output size,
 * transformed, multiplied point by point, transformed back, each image transformed once for all
 * filters).  Same arguments, same result up to rounding (fp32 throughout).  Padded sides are the
 * next powers of two: the full-convolution size (Ho + R - 1) x (Wo + S - 1) must not exceed
 * 64 x 64, else DLL_ERR_UNSUPPORTED (and a workspace size of 0); within that, filters may be
 * larger than the direct kernels take (R * S > 144).  ws holds the spectra:
 * dll_conv_full_fft_workspace_bytes(d) bytes, device memory, caller-owned, overwritten. */
size_t dll_conv_full_fft_workspace_bytes(const dll_conv_desc *d);
dll_status dll_conv_full_bwd_fft(const dll_conv_desc *d, const float *dy, const float *y,
                                 const unsigned char *pool_idx, const float *w, float *dx, void *ws,
                                 size_t ws_bytes, void *stream);

/* Filter-gradient layer (Section II-A, gradient computations):
 *   dw[k,c,r,s] = sum_{n,i,j} dz[n,k,i,j] * xpad[n,c,i+r,j+s];  dbias[k] = sum_{n,i,j} dz[n,k,i,j]
 * with dz as above (same rules for y and pool_idx).  dbias may be NULL.  The batch reduction is a fixed-order tree:
 * results are bit-identical from run to run. */
dll_status dll_conv_valid_wgrad(const dll_conv_desc *d, const float *x, const float *dy,
                                const float *y, const unsigned char *pool_idx, float *dw,
                                float *dbias, void *ws, size_t ws_bytes, void *stream);

/* The two launches of dll_conv_valid_wgrad as calls of their own, for callers that gather the
 * reductions of several layers behind their filter-gradient kernels (the training step below does
 * that with its closing launch) or that time the kernel alone.  _partial runs the filter-gradient
 * kernel: it leaves the per-workgroup partial sums of dw and dbias in ws (same size as above,
 * layout private to the library) and writes nothing else.  _finish adds them up in the fixed
 * order and writes dw (and dbias unless NULL); it reads ws as the _partial call of the SAME
 * descriptor left it, on the same stream or after it.  The two in a row give bit for bit what
 * dll_conv_valid_wgrad gives.  Errors as there; dw == ws -> DLL_ERR_SHAPE. */
dll_status dll_conv_valid_wgrad_partial(const dll_conv_desc *d, const float *x, const float *dy,
                                        const float *y, const unsigned char *pool_idx, void *ws,
                                        size_t ws_bytes, void *stream);
dll_status dll_conv_valid_wgrad_finish(const dll_conv_desc *d, float *dw, float *dbias,
                                       const void *ws, size_t ws_bytes, void *stream);

/* The same filter-gradient layer for callers that cannot allocate device memory or carry a
 * workspace: code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments (minus the workspace), same kernels, bit-identical results; the partial sums
 * live in an array built into the library, DLL_NOALLOC_SCRATCH_BYTES of device memory that every
 * GPU the library runs on holds until the process ends.  The call allocates and frees nothing.
 *   - A layer whose dll_conv_workspace_bytes(d) exceeds DLL_NOALLOC_SCRATCH_BYTES is rejected
 *     with DLL_ERR_SCRATCH_LIMIT before anything is launched (config 5's largest layer needs 3.7 MB).
 *   - All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (two
 *     streams, two threads) race and give undefined results; calls on one stream are ordered.
 *     Nothing in the array has to be cleared between calls.
 *   - The first call on a device asks the runtime for the array's address on that device; make
 *     that first call outside graph capture. */
#define DLL_NOALLOC_SCRATCH_BYTES ((size_t)8 << 20)
dll_status dll_conv_valid_wgrad_noalloc(const dll_conv_desc *d, const float *x, const float *dy,
                                        const float *y, const unsigned char *pool_idx, float *dw,
                                        float *dbias, void *stream);

/* One CD-1 step of a convolutional RBM with binary visible and hidden units (Section II:
 * RBM/CRBM trained with Contrastive Divergence).  d->act and d->pool are ignored.
 *   h0p = sigmoid(b_hid[k] + valid(v0, W));   h0s = 1[uniform < h0p]   (or h0_sample_in)
 *   v1  = sigmoid(c_vis[ch] + full(h0s, W));  h1p = sigmoid(b_hid[k] + valid(v1, W))
 *   dW = (grad(v0,h0p) - grad(v1,h1p)) / N;   db[k] = sum(h0p - h1p) / N;
 *   dc[ch] = sum(v0 - v1) / N;                recon_mse = mean((v0 - v1)^2)
 *   lr != 0:  W += lr*dW, b_hid += lr*db, c_vis += lr*dc   (after all gradients are formed)
 * uniform [N][K][Ho][Wo] in [0,1) is required unless h0_sample_in is given.  dW, db, dc are
 * required; h0_prob, h0_sample, v1, h1_prob and recon_mse (device scalar) may be NULL. */
size_t dll_crbm_workspace_bytes(const dll_conv_desc *d);
dll_status dll_crbm_cd1_step(const dll_conv_desc *d, const float *v0, float *W, float *b_hid,
                             float *c_vis, const float *uniform, const float *h0_sample_in,
                             float lr, float *dW, float *db, float *dc, float *h0_prob,
                             float *h0_sample, float *v1, float *h1_prob, float *recon_mse,
                             void *ws, size_t ws_bytes, void *stream);

/* The CD-1 step with a choice of visible unit and of hidden layer (Section II: the RBM's unit
 * types; the CRBM's second version with probabilistic max pooling).  Everything not said here
 * is as in dll_crbm_cd1_step, which is this call with (DLL_VISIBLE_BINARY, hidden_pool 1).
 *   visible  DLL_VISIBLE_BINARY:   v1 = sigmoid(c_vis[ch] + full(h0s, W))
 *            DLL_VISIBLE_GAUSSIAN: v1 = c_vis[ch] + full(h0s, W)   (unit variance; the mean)
 *   hidden_pool 1: independent binary hidden units, uniform [N][K][Ho][Wo]
 *   hidden_pool 2: probabilistic max pooling over 2x2 blocks (Ho and Wo even, else
 *            DLL_ERR_SHAPE): with I = b_hid[k] + valid(v, W), P(h_i = 1) = exp(I_i) /
 *            (1 + sum over the block of exp(I_j)); at most one unit of a block is on.
 *            uniform [N][K][Ho/2][Wo/2] holds one number u per block: with the block's
 *            probabilities q0..q3 (order 2a+b) and fp32 running sums s_i = s_(i-1) + q_i,
 *            unit i is on iff s_(i-1) <= u < s_i, none when u >= s_3.
 *            pool_prob (nullable; must be NULL when hidden_pool is 1) [N][K][Ho/2][Wo/2]
 *            receives P(pooling unit on | v0) = q0 + q1 + q2 + q3. */
dll_status dll_crbm_cd1_step_units(const dll_conv_desc *d, int visible, int hidden_pool,
                                   const float *v0, float *W, float *b_hid, float *c_vis,
                                   const float *uniform, const float *h0_sample_in, float lr,
                                   float *dW, float *db, float *dc, float *h0_prob,
                                   float *h0_sample, float *pool_prob, float *v1, float *h1_prob,
                                   float *recon_mse, void *ws, size_t ws_bytes, void *stream);

/* One CD-1 step of a fully-connected RBM (Section II: RBM trained with Contrastive
 * Divergence; Section II-A: every dense product is one matrix-matrix multiplication).
 *   v0 [batch][n_vis], W [n_hid][n_vis], b_hid [n_hid], c_vis [n_vis], uniform [batch][n_hid]
 *   h0p = sigmoid(b_hid + v0 W^T);  h0s = 1[uniform < h0p]  (or h0_sample_in)
 *   v1  = sigmoid(c_vis + h0s W)  (DLL_VISIBLE_BINARY)  or  c_vis + h0s W  (DLL_VISIBLE_GAUSSIAN)
 *   h1p = sigmoid(b_hid + v1 W^T)
 *   dW = (h0p^T v0 - h1p^T v1) / batch;  db = colsum(h0p - h1p) / batch;
 *   dc = colsum(v0 - v1) / batch;  recon_mse = mean((v0 - v1)^2)
 *   lr != 0:  W += lr*dW, b_hid += lr*db, c_vis += lr*dc   (after all gradients are formed)
 * All pointers are device pointers, 16-byte aligned.  dW, db, dc are required; h0_prob,
 * h0_sample, v1, h1_prob [same shapes as above] and recon_mse (device scalar) may be NULL.
 * Returns DLL_ERR_WORKSPACE when ws is smaller than dll_rbm_workspace_bytes says. */
size_t dll_rbm_workspace_bytes(int batch, int n_vis, int n_hid);
dll_status dll_rbm_cd1_step(int batch, int n_vis, int n_hid, int visible, const float *v0,
                            float *W, float *b_hid, float *c_vis, const float *uniform,
                            const float *h0_sample_in, float lr, float *dW, float *db, float *dc,
                            float *h0_prob, float *h0_sample, float *v1, float *h1_prob,
                            float *recon_mse, void *ws, size_t ws_bytes, void *stream);

/* One mini-batch gradient-descent step of a CNN (Sections II, IV-B, V, VI): forward
 * through every layer, softmax cross-entropy averaged over the batch, backward (full
 * convolutions for the data gradients except into the network input, filter gradients,
 * dense products with the transposed weights), then theta <- theta - lr * grad.
 *   params  host array of 2*(n_conv+n_dense) device pointers: conv w0,b0,w1,b1,... then
 *           dense W0,b0,...; updated in place when lr != 0
 *   grads   NULL, or a host array in the same order; each non-NULL entry receives that
 *           gradient (taken at the parameters as they were on entry)
 *   labels  [N] int32 in [0, classes)
 *   loss    device scalar, required;  logits [N][classes], may be NULL
 *   pool_idx  NULL, or a host array of n_conv device pointers (entries may be NULL): each
 *           non-NULL entry of a pooled layer receives that layer's pooling indices, in the
 *           encoding dll_conv_valid_fwd writes */
size_t dll_cnn_workspace_bytes(const dll_net_desc *net);
dll_status dll_cnn_train_step(const dll_net_desc *net, float *const *params, float *const *grads,
                              const float *x, const int *labels, float lr, float *loss,
                              float *logits, unsigned char *const *pool_idx, void *ws,
                              size_t ws_bytes, void *stream);

/* The same step with momentum and weight decay (Section II names both as learning options,
 * Section IV trains with momentum 0.9).  Reading taken here, the classical form, per parameter:
 *   v <- momentum * v - lr * (g + weight_decay * theta);   theta <- theta + v
 * with weight_decay applied to filters and dense weights only (0 for biases).
 *   velocity  host array of device pointers, same order and shapes as params; required, updated
 *             in place when lr != 0 (start from zeros)
 * Everything else as in dll_cnn_train_step, which equals momentum = weight_decay = 0. */
dll_status dll_cnn_train_step_momentum(const dll_net_desc *net, float *const *params,
                                       float *const *velocity, float *const *grads, const float *x,
                                       const int *labels, float lr, float momentum,
                                       float weight_decay, float *loss, float *logits,
                                       unsigned char *const *pool_idx, void *ws, size_t ws_bytes,
                                       void *stream);

/* Inference pass of the same network description (Sections IV-VI: the networks the paper times
 * end in a softmax layer): the convolution blocks, the dense layers (the last one without
 * activation) and the softmax of its outputs.  Nothing is kept for a backward pass: activations
 * ping-pong between two workspace buffers and no pooling index is written.
 *   params  host array of 2*(n_conv+n_dense) device pointers, order as in dll_cnn_train_step; read only
 *   x       [N][C][H][W] of the first layer
 *   logits  [N][classes], may be NULL;  prob [N][classes], may be NULL (not both)
 * Errors as for dll_cnn_train_step. */
size_t dll_cnn_forward_workspace_bytes(const dll_net_desc *net);
dll_status dll_cnn_forward(const dll_net_desc *net, const float *const *params, const float *x,
                           float *logits, float *prob, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------------------
 * Operators of large language models, beside the dense layers, the loss and the update of the
 * network steps above: a gated feed-forward block, attention, softmax cross entropy over a large
 * vocabulary, and clipping by the global gradient norm with the momentum step behind it.
 * The conventions at the top hold: device pointers, row-major and contiguous, 16-byte aligned
 * (else DLL_ERR_SHAPE) unless stated (labels, row_loss, row_lse, loss and norm: to 4 bytes),
 * caller-owned workspaces, errors before any launch.
 * Tensors typed `void *` hold the descriptor's dtype.  Sums, softmax statistics and norms are
 * taken in 32 bits or more; with DLL_BF16 what one product hands to the next is rounded to
 * bfloat16 once (to nearest; the loss's probabilities once as exponentials and once more as they
 * enter the gradients' products), and results are rounded once.  At most 2^24 tokens and 2^20
 * features, hidden units or classes; a tensor of 2^31 or more elements -> DLL_ERR_UNSUPPORTED.
 * The same call gives the same bits on every run.  Nothing is allocated on the device or copied
 * from the host, so every call can be captured into a graph (calls that overlap in time need
 * workspaces of their own).  bfloat16 rows of odd length are copied into the workspace first,
 * unless there are few of them to multiply with.  Products of DLL_FP32 tensors may be taken on
 * three bfloat16 parts of each number: errors are those of single precision, but numbers below
 * 2^-110 lose digits; where a tile's sums are not finite it is taken again without the parts,
 * so an infinity or a NaN in one row may change its neighbours' last digits, and nothing more.
 * ------------------------------------------------------------------------------------- */
typedef enum { DLL_FP32 = 0, DLL_BF16 = 1 } dll_dtype;

/* The gate's activation: identity, sigmoid, max(a, 0), a * sigmoid(a), a * Phi(a) with Phi the
 * normal distribution's cumulative function (not its tanh approximation). */
typedef enum { DLL_GATE_IDENTITY = 0, DLL_GATE_SIGMOID = 1, DLL_GATE_RELU = 2, DLL_GATE_SILU = 3, DLL_GATE_GELU = 4 } dll_gate;

typedef struct {
  int tokens, width, hidden;
  int gate;  /* dll_gate */
  int dtype; /* dll_dtype of all tensors */
} dll_gated_desc;

/* Gated feed-forward block over a batch of tokens:
 *   a = x w_gate^T,  b = x w_up^T,  h = act(a) * b,  y = h w_down^T
 *   x, y [tokens][width];  w_gate, w_up [hidden][width];  w_down [width][hidden]
 * gate_pre and up_pre [tokens][hidden] receive a and b, which the backward pass needs (both or
 * neither; NULL in an inference pass).  With DLL_BF16 they are rounded, so the gradients are off by
 * twice what rounding the results alone would leave (3.5e-3 against 1.7e-3, relative). */
size_t dll_gated_fwd_workspace_bytes(const dll_gated_desc *d);
dll_status dll_gated_fwd(const dll_gated_desc *d, const void *x, const void *w_gate, const void *w_up,
                         const void *w_down, void *y, void *gate_pre, void *up_pre, void *ws,
                         size_t ws_bytes, void *stream);

/* Its backward pass, dy [tokens][width] the gradient w.r.t. y:
 *   dh = dy w_down,  da = dh * b * act'(a),  db = dh * act(a)   (act'(0) = 0 for DLL_GATE_RELU)
 *   dx = da w_gate + db w_up,  dw_gate = da^T x,  dw_up = db^T x,  dw_down = dy^T h
 * dx, dw_gate, dw_up and dw_down may each be NULL (that gradient is not taken), not all four. */
size_t dll_gated_bwd_workspace_bytes(const dll_gated_desc *d);
dll_status dll_gated_bwd(const dll_gated_desc *d, const void *x, const void *w_gate, const void *w_up,
                         const void *w_down, const void *gate_pre, const void *up_pre, const void *dy,
                         void *dx, void *dw_gate, void *dw_up, void *dw_down, void *ws, size_t ws_bytes,
                         void *stream);

typedef struct {
  int tokens, width, classes;
  int dtype; /* dll_dtype of x, w, bias and their gradients */
} dll_vocab_desc;

/* Softmax cross entropy of a linear layer over a large vocabulary; its logits are never stored:
 *   z = x w^T + bias,  lse_t = ln sum_v exp z[t][v],  loss_t = lse_t - z[t][labels[t]]
 *   x [tokens][width];  w [classes][width];  bias [classes], may be NULL;  labels [tokens] int32
 * Rows whose label lies outside [0, classes) (padding) do not count: their row_loss and row_lse are
 * 0 and nothing of what x holds there is used.  *loss is the mean over the rows that count, 0 if
 * none does.  row_loss and row_lse [tokens] fp32 may be NULL.  A bias of -infinity takes a class out;
 * logits that are NaN or +infinity, or a row without a finite one, give a loss of NaN. */
size_t dll_vocab_loss_fwd_workspace_bytes(const dll_vocab_desc *d);
dll_status dll_vocab_loss_fwd(const dll_vocab_desc *d, const void *x, const void *w, const void *bias,
                              const int *labels, float *row_loss, float *row_lse, float *loss, void *ws,
                              size_t ws_bytes, void *stream);

/* The same with the gradients of scale * loss:
 *   dz = scale / count * (softmax(z) - onehot(labels)),  dx = dz w,  dw = dz^T x,  dbias = sum_t dz
 * dx rows that do not count are 0.  dx, dw and dbias may each be NULL (not all three; dbias needs bias).
 * exp(z) is kept for a piece of the tokens at a time, 1 GiB at most. */
size_t dll_vocab_loss_grad_workspace_bytes(const dll_vocab_desc *d);
dll_status dll_vocab_loss_grad(const dll_vocab_desc *d, const void *x, const void *w, const void *bias,
                               const int *labels, float scale, float *row_loss, float *row_lse,
                               float *loss, void *dx, void *dw, void *dbias, void *ws, size_t ws_bytes,
                               void *stream);

/* A list of n tensors, as host arrays that are read during the call only: their numbers of elements
 * (0 is allowed) and types. */
typedef struct {
  int n;
  const size_t *counts;
  const int *dtypes; /* dll_dtype of each gradient */
} dll_tensor_list;

/* The 2-norm over all elements of all gradients, *norm a device scalar.  grads is a host array of n
 * device pointers (aligned to their elements; NULL only where the count is 0); none of them may be norm
 * (-> DLL_ERR_SHAPE).  Squares are added in 64 bits in a fixed order. */
size_t dll_grad_norm_workspace_bytes(const dll_tensor_list *list);
dll_status dll_grad_norm(const dll_tensor_list *list, const void *const *grads, float *norm, void *ws,
                         size_t ws_bytes, void *stream);

/* Clipping by the global norm: out = c * grad with c = min(1, max_norm / norm) in 32 bits, max_norm > 0 (infinity:
 * c = 1), out in the gradients' types; out[i] may be grads[i], but no other gradient, output or norm
 * (-> DLL_ERR_SHAPE).  Where *norm is not finite (more than 32 bits hold, too) c is 1.
 * Workspace as for dll_grad_norm. */
dll_status dll_grad_clip(const dll_tensor_list *list, const void *const *grads, void *const *out,
                         float max_norm, float *norm, void *ws, size_t ws_bytes, void *stream);

/* The momentum step of dll_cnn_train_step_momentum on gradients clipped in passing (they are not written):
 *   v <- momentum * v - lr * (c * g + weight_decay * theta);   theta <- theta + v
 * params and velocity are host arrays of n fp32 device pointers; weight_decay a host array of n factors,
 * or NULL (none).  copies, or NULL, is a host array of n device pointers (each may be NULL) that receive
 * the new parameters in bfloat16.  No tensor may be listed twice among the three, nor be a gradient or
 * norm (-> DLL_ERR_SHAPE).  Where *norm is not finite no step is taken: only *norm is written. */
dll_status dll_momentum_update_clipped(const dll_tensor_list *list, float *const *params,
                                       float *const *velocity, const void *const *grads, float lr,
                                       float momentum, const float *weight_decay, float max_norm,
                                       float *norm, void *const *copies, void *ws, size_t ws_bytes,
                                       void *stream);

typedef struct {
  int q_tokens, kv_tokens;       /* rows of q and o; of k and v */
  int sequences;                 /* packed into them */
  int heads, kv_heads, head_dim; /* heads a multiple of kv_heads; head_dim at most 256 */
  int causal;                    /* 0 or 1 */
  int dtype;                     /* dll_dtype of all tensors but lse */
  int q_row, kv_row;             /* elements from a token's row to the next; 0: heads * head_dim, kv_heads * head_dim */
} dll_attention_desc;

/* Attention of packed sequences.  Sequence s has the tokens q_starts[s] to q_starts[s + 1] of q and kv_starts[s] to
 * kv_starts[s + 1] of k and v, n_q and n_k of them (either may be 0; both arrays [sequences + 1] int32 on the device, not
 * decreasing; they may be the same one).  Head h reads the keys and values of head h / (heads / kv_heads):
 *   s_ij = scale q_i . k_j for the keys that query i may see: all of its sequence, with causal those with j <= i + n_k - n_q
 *   lse_i = ln sum_j exp s_ij,  p_ij = exp(s_ij - lse_i),  o_i = sum_j p_ij v_j
 *   q [q_tokens][heads][head_dim] in rows of q_row elements, k and v [kv_tokens][kv_heads][head_dim] in rows of kv_row
 *   (so that one projection's output may hold all three), at any multiple of their elements
 *   o [q_tokens][heads][head_dim] contiguous;  lse [heads][q_tokens] fp32, may be NULL
 * A query that may see no key has o = 0 and lse = -infinity.  Rows outside the sequences are neither read nor written.  What other
 * sequences hold does not matter, and what keys, values, queries and d_o hold that is not finite reaches the results of those that see them
 * or are seen by them alone (as NaN, where they would be infinite, too, and in any elements of their rows).  scale is at most 2^127 in size
 * (else DLL_ERR_SHAPE); q_i . k_j and s_ij count as infinite from 2.3e38 on.  Starts outside [0, tokens] are taken as the nearest of these.  With
 * DLL_BF16 p is rounded, relative to its row's maximum, before it meets v.  Products of DLL_FP32 tensors are taken on three bfloat16 parts of each number, here without a second
 * pass: numbers from 3.39e38 on count as infinite.  (q_tokens / 32 + sequences) * heads, and the same of kv_tokens, at most 2^24 - 1. */
size_t dll_attention_fwd_workspace_bytes(const dll_attention_desc *d);
dll_status dll_attention_fwd(const dll_attention_desc *d, const void *q, const void *k, const void *v,
                             const int *q_starts, const int *kv_starts, float scale, void *o, float *lse,
                             void *ws, size_t ws_bytes, void *stream);

/* Its backward pass, d_o [q_tokens][heads][head_dim] the gradient w.r.t. o, from o and lse as the forward pass left them:
 *   delta_i = d_o_i . o_i,  ds_ij = p_ij (d_o_i . v_j - delta_i)
 *   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij d_o_i   (over the heads that read j, too)
 * dq in rows like q's, dk and dv in rows like k's; each may be NULL (that gradient is not taken), not all three.  A key that no
 * query may see has gradients of 0.  With DLL_BF16 p and ds are rounded before the sums, and delta takes o as it was rounded, but for queries that
 * see few keys. */
size_t dll_attention_bwd_workspace_bytes(const dll_attention_desc *d);
dll_status dll_attention_bwd(const dll_attention_desc *d, const void *q, const void *k, const void *v,
                             const int *q_starts, const int *kv_starts, float scale, const void *o,
                             const float *lse, const void *d_o, void *dq, void *dk, void *dv, void *ws,
                             size_t ws_bytes, void *stream);

/* A cache of keys and values in pages that requests take as they grow.  k_cache and v_cache [pages][kv_heads][page_tokens][head_dim],
 * 16-byte aligned, may have 2^31 or more elements; token t of request r is place t % page_tokens of page
 * table[r][t / page_tokens].  At most 2^16 requests; fewer than 2^31 tokens in all pages, 2^30 in a row of the table. */
typedef struct {
  int requests;
  int heads, kv_heads, head_dim; /* heads a multiple of kv_heads; head_dim at most 256 */
  int pages, page_tokens;        /* of the cache */
  int table_pages;               /* columns of the table */
  int dtype;                     /* dll_dtype of all tensors but lse */
} dll_cache_desc;

/* Pages and slots for a step's new tokens, all int32:
 *   lengths [requests]  tokens of each request, the new ones among them;  added [requests]  how many of these are new (below 0
 *           counts as 0, more than lengths as lengths)
 *   free_pages [n_free] pages that nobody has, taken from entry *free_at on (NULL: 0; n_free = 0: free_pages may be NULL) in the requests' order
 *   table   [requests][table_pages]  entries of the pages that the requests had before are read, those of the new pages are written,
 *           the others left as they are
 *   starts  [requests + 1]  receives where each request's new tokens lie when they are packed (q_starts of dll_attention_fwd); sums
 *           stop at 2^30, and so do those of state
 *   slots   [tokens]  receives page * page_tokens + place for each new token; -1 where it has no page.  tokens, at least 1, is the array's room:
 *           new tokens behind it get neither slot nor table entry; what lies behind the new tokens is left as it is
 *   state   [2]  receives the first entry of free_pages that is still free, and how many pages were missing, as the list was too short (their
 *           entries are -1) or the table too narrow
 * Calls may be repeated: they change none of what they read. */
dll_status dll_cache_plan(const dll_cache_desc *d, const int *lengths, const int *added, const int *free_pages,
                          int n_free, const int *free_at, int *table, int *starts, int *slots, int tokens,
                          int *state, void *stream);

/* Rows of new tokens into the cache: k and v [tokens][kv_heads][head_dim] in rows of `row` elements (0: contiguous), at any multiple of their
 * elements; slots [tokens] int32 as dll_cache_plan leaves them.  Tokens whose slot lies outside [0, pages * page_tokens) are left out.
 * Slots that are not -1 have to differ. */
dll_status dll_cache_write(const dll_cache_desc *d, int tokens, int row, const void *k, const void *v,
                           const int *slots, void *k_cache, void *v_cache, void *stream);

/* Attention of one new token a request over its keys and values in the cache, its own among them:
 *   o[r][h] = sum_t p_t v_t,  p = softmax_t(scale q[r][h] . k_t),  t < lengths[r], keys and values of head h / (heads / kv_heads)
 *   q, o [requests][heads][head_dim];  table [requests][table_pages], lengths [requests] int32;  lse [requests][heads] fp32, may be NULL
 * A length below 0 counts as 0, one that the table has no room for as that room.  Keys whose table entry lies outside [0, pages)
 * are left out, and nothing that pages hold behind a request's last token is used.  A request without keys has o = 0 and lse = -infinity.  What keys
 * and values hold that is not finite reaches the outputs of the heads that read it alone; a key whose score is -infinity has no weight.
 * scale as for dll_attention_fwd.  With DLL_BF16 p meets v in two parts of that type. */
size_t dll_paged_attention_workspace_bytes(const dll_cache_desc *d);
dll_status dll_paged_attention(const dll_cache_desc *d, const void *q, const void *k_cache, const void *v_cache,
                               const int *table, const int *lengths, float scale, void *o, float *lse, void *ws,
                               size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
