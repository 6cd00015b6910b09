/*
 * nf — the per-layer local training step of adaptive local learning on one AMD MI355X
 * (gfx950), as a C-ABI library of hand-written HIP kernels.
 *
 * Method: NeuroFlux (arXiv 2402.14139).  One local step is the body of Algorithm 2 for
 * one (batch, layer) pair:
 *     x_{n+1} = ReLU(P_n(theta_n * x_n))                         Eq. 1
 *     z       = gamma_n F_n beta_n x_{n+1}                       Eq. 2
 *     L       = mean_k CE(z_k, y_k)                              Eq. 3
 *     gradients of L w.r.t. (theta_n, beta_n, gamma_n) only, then the update,
 * plus the activation cache that carries a trained block's output to the next block at
 * that block's own batch size (section "Efficient Forward Propagation via Prefetching and
 * Adaptive Batching").
 *
 * ---- Data layout (all tensors dense fp32 unless stated, all pointers DEVICE pointers) ----
 *   activations  NHWC : x[n][h][w][c]
 *   conv weights KRSC : W[k][r][s][c]         (k = output channel)
 *   projection        : Wp[k][c]              (1x1, stride skip_stride, no bias)
 *   aux conv     ARSK : Wa[a][r][s][k]        (a = aux filter, k = layer output channel)
 *   linear            : Wf[q][f], f = (i*pool_ow + j)*A + a   (NHWC flatten of the pooled map)
 *   labels            : int32 in [0, n_classes)
 *   cache row         : one sample's emitted activation, H*W*C contiguous floats (NHWC)
 * These are index permutations of the paper-notation tensors (NCHW / OIHW / flatten a,i,j);
 * the library never transposes activations.
 *
 * ---- Ownership, streams, errors -----------------------------------------------------------
 *   The caller owns every buffer, including the workspace `ws` (size from
 *   nf_workspace_bytes, 256-byte aligned).  The library allocates nothing and keeps no
 *   state between calls (five documented exceptions: the static scratch array of
 *   nf_local_step_static, the event pool of the prefetch mode of nf_block_train_epoch, the
 *   graph handles of nf_block_graph_create, the process-wide contraction mode of nf_contraction,
 *   and the measurement aid nf_prof_begin/end).  `stream` is a hipStream_t passed as void*
 *   (NULL = default stream); every call only enqueues work on it and never synchronises the host.
 *   Every device pointer must be 16-byte aligned.
 *   Every call returns NF_OK (0) or a negative nf_status.  Arguments are validated before
 *   anything is enqueued, so a failing call has no side effects on device memory.
 *   Labels outside [0,n_classes) and cache indices outside [0,capacity) are NOT detected
 *   (they are data on the device); such a label contributes as if no class matched and
 *   such an index is clamped into range.
 *   Calls sharing a workspace must be ordered on one stream.
 *   Values that are not finite: an infinity in the input or the weights reaches the results whose sum holds
 *   it.  A window that lies partly over the zero padding, with an infinite or NaN weight there (or, in a
 *   weight gradient, an infinite gradient beside the padding), is the exception: kernels that leave the padding
 *   out (the 3x3 minimal filtering, and the direct kernels on small maps, by sizes and batch) do not see it, the
 *   others form 0 * inf = NaN there, which a ReLU makes 0.
 */
#ifndef NF_H
#define NF_H
#include <stddef.h>
#include <stdint.h>
#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  NF_OK = 0,
  NF_ERR_NULL = -1,        /* a required pointer is NULL                                   */
  NF_ERR_BAD_DESC = -2,    /* non-positive size, inconsistent shapes, misaligned pointer   */
  NF_ERR_UNSUPPORTED = -3, /* filter/stride/pool outside what the kernels implement        */
  NF_ERR_WORKSPACE = -4,   /* workspace NULL, misaligned or smaller than required          */
  NF_ERR_CACHE_RANGE = -5, /* first + B exceeds the cache capacity                         */
  NF_ERR_DEVICE = -6,      /* a HIP call failed (launch error)                             */
  NF_ERR_SCRATCH_LIMIT = -7 /* nf_local_step_static: the step needs more than NF_STATIC_SCRATCH_BYTES */
} nf_status;

/* Layer n of Eq. 1: conv theta_n (+bias, + optional shortcut), ReLU, optional max-pool P_n.
 * Supported: 1 <= R,S <= 15, 1 <= stride <= 4, 0 <= pad < R + S; max-pool with
 * 2*pool_pad <= pool_k <= 15 and any positive stride.  Anything else: NF_ERR_UNSUPPORTED. */
typedef struct {
  int32_t C_in, H_in, W_in;
  int32_t C_out, R, S, stride, pad;
  int32_t pool_kind; /* 0 none, 1 max */
  int32_t pool_k, pool_stride, pool_pad;
  int32_t skip_kind; /* 0 none; 1 identity (x_skip has the conv-output shape);
                        2 projection: + sum_c Wp[k][c] * x_skip[n][i*skip_stride][j*skip_stride][c] */
  int32_t skip_C, skip_H, skip_W, skip_stride;
} nf_layer_desc;

/* Auxiliary head A_n of Eq. 2: conv beta_n (R x S, stride 1, pad, + bias, ReLU if relu),
 * adaptive pooling F_n to pool_oh x pool_ow (average or max: the two down-sampling mechanisms
 * the text below Eq. 1 names), linear gamma_n to n_classes.  The loss l of Eq. 3 is softmax
 * cross-entropy, or the mean squared error against the one-hot label (mean over the classes,
 * then over the batch).  C_in/H_in/W_in describe the tensor the layer emits (post-pool). */
enum { NF_HEAD_POOL_AVG = 0, NF_HEAD_POOL_MAX = 1 };
enum { NF_LOSS_CE = 0, NF_LOSS_MSE = 1 };
typedef struct {
  int32_t C_in, H_in, W_in;
  int32_t A, R, S, pad, relu;
  int32_t pool_oh, pool_ow;
  int32_t n_classes;
  int32_t head_pool; /* NF_HEAD_POOL_*; ties of the max go to the first element in row-major order */
  int32_t loss_kind; /* NF_LOSS_* */
} nf_aux_desc;

typedef struct {
  float lr, momentum;
} nf_sgd_desc;

/* Parameters of the layer (theta_n) and of its head (beta_n, gamma_n).  The same structs
 * carry gradients and momentum buffers.  Wp is ignored unless skip_kind == 2. */
typedef struct {
  float *W, *b, *Wp;
} nf_layer_params;
typedef struct {
  float *Wa, *ba, *Wf, *bf;
} nf_aux_params;

const char *nf_strerror(int32_t status);

/* How the wide contractions (the convolution of Eq. 1 and its weight gradient in Algorithm 2, for
 * layers with at least 128 filters) are carried out.  Operands, results and accumulation are fp32
 * in all modes.
 *   NF_CONTRACT_F32     (default) fp32 matrix-core instructions (v_mfma_f32_*).  3x3 convolutions of
 *                       stride 1 and pad 1, and their weight gradients, go through the minimal filtering
 *                       algorithms F(2x2,3x3) / F(3x3,2x2), all in fp32, where that is faster and its
 *                       error against 64 bits is below the direct sum's.
 *   NF_CONTRACT_BF16X6  each fp32 operand element is cut into three bfloat16 pieces that sum to it
 *                       exactly; six of the nine piece products are accumulated in fp32 by bf16
 *                       matrix-core instructions.  The three left out are together below 2^-21 of
 *                       the product in the worst case and about 2^-24 of it in the root mean
 *                       square, i.e. of the size of an fp32 rounding; over the reductions of this
 *                       library (36 ... 4608 terms) a single result's measured error against fp64
 *                       equals that of the fp32 instructions.  These instructions round their
 *                       running sums down, not to nearest: errors of different results share a
 *                       sign, and averages over the pixels of a 512-channel layer are off by 1.4e-7
 *                       to 1.7e-7, fp32 instructions' by 4e-8; of sums that only grow 2e-6 and 1e-8.
 *                       An operand element that is +-inf gives NaN instead of +-inf.  Weight
 *                       gradients that NF_CONTRACT_F32 carries out faster run as there.
 *   NF_CONTRACT_BF16X9  the same with all nine piece products: every product x*w enters the fp32
 *                       accumulation exactly, as with the fp32 instructions (the running sums are
 *                       rounded as in BF16X6); 1.5x the matrix-core work of BF16X6.
 * Process-wide (read when a call enqueues its kernels); returns the previous mode, or
 * NF_ERR_BAD_DESC for an unknown mode.  mode = -1 only queries. */
enum { NF_CONTRACT_F32 = 0, NF_CONTRACT_BF16X6 = 1, NF_CONTRACT_BF16X9 = 2 };
int32_t nf_contraction(int32_t mode);

/* Emitted sizes: conv output (Ho,Wo) and post-pool (Hp,Wp).  Any out pointer may be NULL. */
int32_t nf_layer_out_dims(const nf_layer_desc *d, int32_t *Ho, int32_t *Wo, int32_t *Hp, int32_t *Wp);

/* Bytes of workspace the calls below want for this (layer, head, batch); single-layer calls also take a
 * smaller one that still holds the direct contraction kernels, and run those where the others do not fit.
 * At most NF_STATIC_SCRATCH_BYTES where that holds the direct kernels.  `a` may be NULL when only
 * nf_layer_fwd will be called. */
int32_t nf_workspace_bytes(const nf_layer_desc *d, const nf_aux_desc *a, int32_t B, size_t *out);

/* Where two intermediates of the step live inside the workspace (byte offset and size), for
 * callers that want to inspect them after nf_aux_fwd_loss / nf_local_step (tests compare the
 * ReLU and max-pool decisions the kernels took):
 *   NF_WS_AUX_ACT   the head's convolution output after its ReLU (Eq. 2, beta_n), fp32
 *                   [B][Hu][Wu][A];
 *   NF_WS_POOL_ARG  one byte per emitted element [B][Hp][Wp][C_out]: index u*pool_k+v of the
 *                   window cell the max-pool P_n of Eq. 1 selected (size 0 when un-pooled);
 *   NF_WS_HEAD_ARG  int32 [B][pool_oh][pool_ow][A]: flat position h*Wu+w inside the head's
 *                   convolution output that a max-pooling F_n selected (size 0 when F_n averages). */
enum { NF_WS_AUX_ACT = 0, NF_WS_POOL_ARG = 1, NF_WS_HEAD_ARG = 2 };
int32_t nf_workspace_region(const nf_layer_desc *d, const nf_aux_desc *a, int32_t B, int32_t which,
                            size_t *offset, size_t *bytes);

/* Eq. 1.  x [B,H_in,W_in,C_in], x_skip per skip_kind (NULL if 0), y OUT [B,Hp,Wp,C_out].
 * Records in ws what the backward needs (pool arg-max). */
int32_t nf_layer_fwd(const nf_layer_desc *d, int32_t B, const float *x, const float *x_skip,
                     const nf_layer_params *p, float *y, void *ws, size_t ws_bytes, void *stream);

/* Eq. 2 + Eq. 3.  y is the emitted activation [B,Hp,Wp,C_out]; *loss_out (device float)
 * receives the batch-mean cross-entropy.  Leaves the head's activations and dL/dz in ws.
 * `d` is the layer the head is attached to (it fixes where the head's data sits in ws). */
int32_t nf_aux_fwd_loss(const nf_layer_desc *d, const nf_aux_desc *a, int32_t B, const float *y,
                        const int32_t *labels, const nf_aux_params *ap, float *loss_out, void *ws,
                        size_t ws_bytes, void *stream);

/* Algorithm 2, gradient line: gradients of the local loss w.r.t. theta_n, beta_n, gamma_n.
 * Must follow nf_layer_fwd and nf_aux_fwd_loss on the same ws.  gp/ga are OVERWRITTEN
 * (not accumulated).  No gradient is formed for x or x_skip. */
int32_t nf_local_bwd_wgrad(const nf_layer_desc *d, const nf_aux_desc *a, int32_t B,
                           const float *x, const float *x_skip, const float *y,
                           const nf_layer_params *p, const nf_aux_params *ap,
                           const nf_layer_params *gp, const nf_aux_params *ga, void *ws,
                           size_t ws_bytes, void *stream);

/* Algorithm 2, update line, for n_tensors (<= 16) tensors in one launch:
 *   v = momentum*v + g ; w = w - lr*v      (v == NULL or momentum == 0: w = w - lr*g)
 * w, g, v are HOST arrays of device pointers; numel a HOST array of element counts. */
int32_t nf_sgd_update(const nf_sgd_desc *s, int32_t n_tensors, float *const *w, const float *const *g,
                      float *const *v, const int64_t *numel, void *stream);

/* Updates made orthogonal.  A matrix G [rows][cols], dense, goes through `steps` Newton-Schulz steps,
 *   X = G / (|G| + eps), |G| the root of the sum of squares;  X <- a X + (b A + c A^2) X with A = X X^T (rows <= cols; else X^T X),
 * step k with a[k], b[k], c[k].  They drive the singular values towards those that the polynomial x (a + b x^2 + c x^4) repeats.  Products keep 22 bits of their
 * operands and sums are fp32, as errors of small singular values grow by the a's product.  The bound of every step's results, where the singular values
 * begin at most at 1, has to lie between 1e-6 and 1e9 (or to be 0: a = b = c = 0): else NF_ERR_UNSUPPORTED.  1 <= steps <= NF_ORTH_STEPS, eps >= 0.
 * n_matrices (<= NF_ORTH_MATRICES) share the launches; rows, cols, and the arrays of device pointers are HOST arrays.  rows, cols <= 2^20, the lesser of them
 * <= 2^14.  A matrix with an infinity or a NaN gives NaN throughout, and so does one of zeros where eps is 0. */
#define NF_ORTH_STEPS 12
#define NF_ORTH_MATRICES 32
typedef struct {
  int32_t steps;
  float eps, a[NF_ORTH_STEPS], b[NF_ORTH_STEPS], c[NF_ORTH_STEPS];
} nf_orth_desc;
int32_t nf_orthogonalise_workspace_bytes(const nf_orth_desc *d, int32_t n_matrices, const int32_t *rows,
                                         const int32_t *cols, size_t *out);
/* y = the last X, in G's type (NF_F32, NF_BF16, NF_F16).  A matrix's y may be its g, not another one's; no two y may be the same. */
int32_t nf_orthogonalise(const nf_orth_desc *d, int32_t dtype, int32_t n_matrices, const void *const *g, void *const *y,
                         const int32_t *rows, const int32_t *cols, void *ws, size_t ws_bytes, void *stream);
/* nf_sgd_update for weight matrices, the update made orthogonal (filters [C_out][R][S][C_in] are matrices of C_out rows):
 *   v = momentum v + g;  u = g + momentum v (nesterov != 0) or v;  w = (1 - lr weight_decay) w - lr sqrt(max(1, rows / cols)) X(u)
 * v == NULL or momentum == 0: u = g.  All fp32.  The workspace is nf_orthogonalise's.  No w or v may be
 * another one's, nor a g. */
typedef struct {
  float lr, momentum, weight_decay;
  int32_t nesterov;
  nf_orth_desc orth;
} nf_muon_desc;
int32_t nf_muon_update(const nf_muon_desc *d, int32_t n_matrices, float *const *w, const float *const *g,
                       float *const *v, const int32_t *rows, const int32_t *cols, void *ws, size_t ws_bytes,
                       void *stream);

/* Activation cache.  cache [capacity][sample_elems], cache_labels [capacity] (may be NULL
 * together with labels).  Write stores batch rows at [first, first+B).  Read gathers B rows:
 * idx == NULL -> rows first..first+B-1, else rows idx[0..B) (device int64) — B is the
 * CONSUMING block's batch size and need not equal the batch size used for writing. */
int32_t nf_cache_write(float *cache, int32_t *cache_labels, int64_t capacity, int64_t sample_elems,
                       int64_t first, int32_t B, const float *y, const int32_t *labels, void *stream);
int32_t nf_cache_read(const float *cache, const int32_t *cache_labels, int64_t capacity,
                      int64_t sample_elems, int64_t first, const int64_t *idx, int32_t B, float *x_out,
                      int32_t *labels_out, void *stream);

/* The whole Algorithm 2 body for one (batch, layer): forward, head, loss, gradients, update
 * of p/ap in place, and y_out = the activation emitted with the PRE-update weights (it is
 * the next layer's input).  gp/ga receive the gradients; vp/va are momentum buffers (may be
 * NULL when s->momentum == 0). */
int32_t nf_local_step(const nf_layer_desc *d, const nf_aux_desc *a, const nf_sgd_desc *s, int32_t B,
                      const float *x, const float *x_skip, const int32_t *labels,
                      const nf_layer_params *p, const nf_aux_params *ap, const nf_layer_params *gp,
                      const nf_aux_params *ga, const nf_layer_params *vp, const nf_aux_params *va,
                      float *y_out, float *loss_out, void *ws, size_t ws_bytes, void *stream);

/* nf_local_step for callers that cannot allocate device memory or hand in a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same
 * kernels and bit-for-bit the same results as nf_local_step, but the scratch lives in a
 * file-scope device array of NF_STATIC_SCRATCH_BYTES inside the library (one copy per GPU the
 * library runs on, held until the process ends) instead of a caller workspace.  The call
 * allocates nothing (no hipMalloc / hipFree, no allocating library routine).
 * A (layer, head, B) whose nf_workspace_bytes exceeds NF_STATIC_SCRATCH_BYTES is rejected with
 * NF_ERR_SCRATCH_LIMIT before anything is enqueued (a 512-channel 3x3 layer at batch 512 on 4x4
 * maps needs 89 MiB, the largest layer of the VGG-16-style workload 115 MiB).
 * Every call on a GPU shares that GPU's array: calls that overlap in time on one GPU (two
 * streams, two threads) race; order them on one stream.  The array keeps the previous call's
 * contents, which is harmless: every region is written by the step before it is read.  The
 * intermediates nf_workspace_region describes are not reachable through this entry point. */
#define NF_STATIC_SCRATCH_BYTES (128u << 20)
int32_t nf_local_step_static(const nf_layer_desc *d, const nf_aux_desc *a, const nf_sgd_desc *s, int32_t B,
                             const float *x, const float *x_skip, const int32_t *labels,
                             const nf_layer_params *p, const nf_aux_params *ap, const nf_layer_params *gp,
                             const nf_aux_params *ga, const nf_layer_params *vp, const nf_aux_params *va,
                             float *y_out, float *loss_out, void *stream);

/* ---- a block of consecutive local layers (the paper's partition of the network into blocks,
 * each trained at its own batch size; Worker loop of Algorithm 2; "Efficient Forward Propagation
 * via Prefetching and Adaptive Batching") ---------------------------------------------------------
 * All arrays are HOST arrays with n_layers entries; the pointers inside the parameter structs
 * are device pointers.  Layer n+1 reads what layer n emits, so its C_in/H_in/W_in must equal
 * layer n's C_out/Hp/Wp.  skip_src (NULL = no shortcuts) gives per layer -1, or the position
 * m <= n of the layer whose INPUT tensor is layer n's shortcut (0 = the block's input batch);
 * that tensor's shape must equal the layer's skip_C/skip_H/skip_W.  aux/ap/gp/ga are not read by
 * nf_block_fill_cache and may be NULL there; vp/va may be NULL when momentum == 0.  gp/ga are
 * scratch of the pass (they hold the last batch's gradients afterwards).  The block calls validate
 * every descriptor, shape, pointer and alignment of every layer before the first enqueue, so an
 * argument error has no side effects; only a HIP error (NF_ERR_DEVICE) can surface mid-pass, and
 * then the prefetch stream, if any, is joined back into `stream` before the call returns. */
typedef struct {
  int32_t n_layers;
  const nf_layer_desc *layers;
  const nf_aux_desc *aux;
  const int32_t *skip_src;
  const nf_layer_params *p;
  const nf_aux_params *ap;
  const nf_layer_params *gp;
  const nf_aux_params *ga;
  const nf_layer_params *vp;
  const nf_aux_params *va;
} nf_block;

/* Workspace of the two block calls at batch size B: two input batches (double buffer), every
 * layer's emitted batch, and the largest single-layer workspace.  It serves smaller batches too, also where
 * those would ask for more (the kernels planned for them want more scratch; they take those that fit, and a call
 * takes what a larger workspace holds beyond this).  In a block without heads the direct kernels of a small last
 * batch, whose reductions are split, may need more than this: the call then returns NF_ERR_WORKSPACE before it
 * enqueues anything. */
int32_t nf_block_workspace_bytes(const nf_block *blk, int32_t B, size_t *out);

/* One pass of the block over n_items cached samples in batches of B (the last one may be
 * smaller): per batch, nf_cache_read (rows idx[j], device int64 [n_items], or rows 0..n_items-1
 * when idx == NULL; cache [capacity][C_in*H_in*W_in of layer 0], cache_labels [capacity]), then
 * nf_local_step layer by layer, each layer handing on the activations it emitted BEFORE its
 * update.  losses (device, [ceil(n_items/B)][n_layers]) receives every local loss.
 * prefetch_stream != NULL: the read of batch j+1 is enqueued there and overlaps the training of
 * batch j (the paper's prefetching); it is ordered after everything already enqueued on `stream`
 * and joined back into `stream` before the call's last batch, so `stream` alone orders the
 * result.  That mode uses four process-wide HIP events per device, created on first use: calls
 * with a prefetch stream must not overlap in time on one device.  Both streams must have the
 * default priority. */
int32_t nf_block_train_epoch(const nf_block *blk, const nf_sgd_desc *s, int32_t B, int64_t n_items,
                             const float *cache, const int32_t *cache_labels, int64_t capacity,
                             const int64_t *idx, float *losses, void *ws, size_t ws_bytes,
                             void *stream, void *prefetch_stream);

/* The same pass (Algorithm 2, the Worker's loop over the batches of a block) as a HIP graph the
 * library captures itself (the per-batch work of a block is a few
 * hundred short launches; replayed from a graph they are enqueued by one call and the gaps between
 * them shrink).  nf_block_graph_create takes the arguments of nf_block_train_epoch without the
 * streams, validates them the same way (same error codes, nothing captured on error), captures the
 * whole pass over the n_items samples on a private stream and instantiates it; *out is the handle.
 * The graph is a snapshot of the ARGUMENTS: every pointer, B, n_items, lr, momentum, the descriptors
 * and the contraction mode in force at creation are fixed; what the pointers point at (cache rows,
 * the index list idx, weights, momentum) is read when the graph runs, so an epoch with a new shuffle
 * is: rewrite idx on the device, launch again.  All buffers must stay alive until the handle is
 * destroyed.  nf_block_graph_launch enqueues one pass on `stream` (default priority) of the device
 * the graph was created on (another current device: NF_ERR_BAD_DESC); results are bit-identical to
 * nf_block_train_epoch with prefetch_stream == NULL.  Launches of one handle must not overlap in
 * time (they share ws).  nf_block_graph_destroy frees the handle (NULL is accepted).  Creation
 * between nf_prof_begin and nf_prof_end is refused with NF_ERR_UNSUPPORTED.  These three calls are
 * the only ones in the library that allocate: the graph objects and the handle, host side. */
typedef struct nf_block_graph nf_block_graph;
int32_t nf_block_graph_create(const nf_block *blk, const nf_sgd_desc *s, int32_t B, int64_t n_items,
                              const float *cache, const int32_t *cache_labels, int64_t capacity,
                              const int64_t *idx, float *losses, void *ws, size_t ws_bytes,
                              nf_block_graph **out);
int32_t nf_block_graph_launch(nf_block_graph *g, void *stream);
int32_t nf_block_graph_destroy(nf_block_graph *g);

/* After the block is trained: forward-only sweep with its final weights over rows [0, n_items)
 * of its input cache in batches of B (last one partial), writing the last layer's emitted
 * activations and the labels to rows [0, n_items) of the next block's cache
 * (cache_out [capacity_out][C_out*Hp*Wp of the last layer]). */
int32_t nf_block_fill_cache(const nf_block *blk, int32_t B, int64_t n_items, const float *cache_in,
                            const int32_t *labels_in, int64_t capacity_in, float *cache_out,
                            int32_t *labels_out, int64_t capacity_out, void *ws, size_t ws_bytes,
                            void *stream);

/* ---- early-exit evaluation ("Trained Output CNN") ---------------------------------------------
 * nf_aux_predict: forward of the head only on emitted activations y [B,Hp,Wp,C_out]; pred_out
 * (device int32 [B]) receives the class with the largest logit (lowest index among equal maxima);
 * with labels, *n_correct (device int32) receives the number of correct predictions of the batch,
 * added to its previous value when accumulate != 0 (labels and n_correct are given together or
 * both NULL); logits_out (device [B][n_classes]) is optional.
 * nf_block_evaluate: the early-exit model that leaves the block after layer exit_layer: rows
 * [0, n_items) of the block's input cache in batches of B (last one partial), forward through
 * layers 0..exit_layer, that layer's head; pred_out [n_items], *n_correct the total (cache_labels
 * and n_correct may both be NULL: plain prediction).  The block's aux and ap arrays are required,
 * gp/ga/vp/va are not read.
 * nf_select_exit (host): index of the exit with the most correct validation predictions; among
 * equals the one whose model has the fewest parameters; among those the earliest. */
int32_t nf_aux_predict(const nf_layer_desc *d, const nf_aux_desc *a, int32_t B, const float *y,
                       const int32_t *labels, const nf_aux_params *ap, int32_t *pred_out, int32_t *n_correct,
                       int32_t accumulate, float *logits_out, void *ws, size_t ws_bytes, void *stream);
int32_t nf_block_evaluate(const nf_block *blk, int32_t exit_layer, int32_t B, int64_t n_items,
                          const float *cache, const int32_t *cache_labels, int64_t capacity,
                          int32_t *pred_out, int32_t *n_correct, void *ws, size_t ws_bytes, void *stream);
int32_t nf_select_exit(int32_t n_exits, const int64_t *n_correct, const int64_t *n_params, int32_t *exit_out);

/* ---- pointwise layers: linear with a fused epilogue, group and layer norm, dropout, a quantised cache ----
 * The operators around a 1x1 layer of channels-last activations, forward and backward, in three types: a
 * dtype of NF_F32, NF_BF16 or NF_F16 is that of the activations and of the weights W; biases, gamma, beta,
 * statistics and the gradients of parameters are fp32.  Products, sums, statistics and activations are formed
 * in fp32 (an activation of a 16-bit type may be off by 8e-6 of its argument) and each result is rounded once.
 * Rows are dense.  Every pointer is 16-byte aligned at its base; rows need no alignment (any K, N, C, cols, n).
 * A workspace of 0 bytes may be NULL.  Outputs must not overlap inputs, but for dropout's y, which may be x or
 * r (and dx, which may be dy).  Results do not depend on the order in which workgroups run. */
enum { NF_F32 = 0, NF_BF16 = 1, NF_F16 = 2 };
/* relu: max(v, 0), its slope at 0 is 0; silu: v / (1 + e^-v); gelu: v Phi(v), Phi the normal distribution's.  At infinities they
 * and their slopes are the limits (inf and 0, 1 and 0). */
enum { NF_ACT_NONE = 0, NF_ACT_RELU = 1, NF_ACT_SILU = 2, NF_ACT_GELU = 3 };

/* D: an element of a row-major matrix is dropped (0) where u < T = rint(65536 p), else scaled by
 * 65536 / (65536 - T).  u(row, col) is the (col % 8)-th half word (low halves first) of Philox4x32-10 (Salmon et
 * al., SC'11) at counter (row * ceil(cols / 8) + col / 8, step), two 64-bit words, with the 64-bit key seed.  The
 * mask is formed again wherever it is needed and never stored; another step gives another mask.  0 <= p, T < 65536. */
typedef struct {
  double p;
  uint64_t seed, step;
} nf_dropout_desc;
/* y = r + D(x) (r may be NULL); backward: dx = D(dy).  rows, cols >= 1, cols < 2^31 - 8, rows * cols < 2^62. */
int32_t nf_dropout_fwd(const nf_dropout_desc *drop, int32_t dtype, int64_t rows, int64_t cols, const void *x,
                       const void *r, void *y, void *stream);
int32_t nf_dropout_bwd(const nf_dropout_desc *drop, int32_t dtype, int64_t rows, int64_t cols, const void *dy,
                       void *dx, void *stream);

/* A layer of N filters on rows of K channels: x [M][K], W [N][K], y [M][N].  1 <= M, N, K, M < 2^31 - 512,
 * K, N <= 2^20, and the tiles of 64 along the longest of M, K, N times those along max(K, N) stay below 2^23. */
typedef struct {
  int32_t dtype, K, N, act;
} nf_linear_desc;
/* Bytes of workspace that the three calls below want at M rows.  They do not grow steadily with M: a sum is cut into other parts at
 * other sizes, and fewer rows may want more.  A buffer for several M holds the largest of their sizes. */
int32_t nf_linear_workspace_bytes(const nf_linear_desc *d, int64_t M, size_t *out);
/* What nf_linear_fwd alone wants: at most that, and often nothing (65536 rows of 512 to 512: 0 and 33.6 MB). */
int32_t nf_linear_fwd_workspace_bytes(const nf_linear_desc *d, int64_t M, size_t *out);
/* z = x W^T + b, y = r + D(act(z)).  b (fp32), r and drop may be NULL; z may be NULL (else it receives the sums before
 * the activation, rounded to the type, which the backward epilogue reads). */
int32_t nf_linear_fwd(const nf_linear_desc *d, int64_t M, const void *x, const void *W, const float *b, const void *r,
                      const nf_dropout_desc *drop, void *y, void *z, void *ws, size_t ws_bytes, void *stream);
/* dz = act'(z) D(dy) and db[n] = sum over the rows of dz before its rounding.  z may be NULL where act is
 * NF_ACT_NONE; drop and db may be NULL. */
int32_t nf_linear_bwd_epilogue(const nf_linear_desc *d, int64_t M, const void *dy, const void *z,
                               const nf_dropout_desc *drop, void *dz, float *db, void *ws, size_t ws_bytes,
                               void *stream);
/* dx = dz W [M][K] in the type, dW = dz^T x [N][K] in fp32.  Either may be NULL (a first layer has no dx; x is not read
 * without dW, nor W without dx), not both. */
int32_t nf_linear_bwd(const nf_linear_desc *d, int64_t M, const void *dz, const void *x, const void *W, void *dx,
                      float *dW, void *ws, size_t ws_bytes, void *stream);

/* Group norm over x [B][HW][C]: C / G neighbouring channels of an image share a mean and a variance.
 * 1 <= B <= 65535, G divides C, C <= 2^16, C / G <= 2048, HW < 2^24, eps >= 0. */
typedef struct {
  int32_t dtype, C, G, act, HW;
  float eps;
} nf_groupnorm_desc;
/* Not steady in B, either: fewer images are cut into more chunks. */
int32_t nf_groupnorm_workspace_bytes(const nf_groupnorm_desc *d, int32_t B, size_t *out);
/* what nf_groupnorm_fwd alone wants */
int32_t nf_groupnorm_fwd_workspace_bytes(const nf_groupnorm_desc *d, int32_t B, size_t *out);
/* y = act((x - mean) rstd gamma + beta), rstd = (var + eps)^-1/2, var the mean square about the mean; mean and rstd
 * [B][G] are written too. */
int32_t nf_groupnorm_fwd(const nf_groupnorm_desc *d, int32_t B, const void *x, const float *gamma, const float *beta,
                         void *y, float *mean, float *rstd, void *ws, size_t ws_bytes, void *stream);
/* With xh = (x - mean) rstd and g = dy act'(xh gamma + beta): dx = rstd (g gamma - avg(g gamma) - xh avg(g gamma xh)),
 * averages over the group; dgamma = sum g xh, dbeta = sum g over images and pixels.  mean and rstd are what the
 * forward wrote. */
int32_t nf_groupnorm_bwd(const nf_groupnorm_desc *d, int32_t B, const void *dy, const void *x, const float *gamma,
                         const float *beta, const float *mean, const float *rstd, void *dx, float *dgamma,
                         float *dbeta, void *ws, size_t ws_bytes, void *stream);

/* Layer norm over the rows of x [M][C].  1 <= M < 2^40, C <= 2^16, eps >= 0. */
typedef struct {
  int32_t dtype, C;
  float eps;
} nf_layernorm_desc;
/* What nf_layernorm_bwd wants for dgamma and dbeta (the forward wants none).  Not steady in M. */
int32_t nf_layernorm_workspace_bytes(const nf_layernorm_desc *d, int64_t M, size_t *out);
/* y = (x - mean) rstd gamma + beta, rstd = (var + eps)^-1/2, var the mean square about the mean.  gamma (else 1) and beta (else 0)
 * may be NULL; mean and rstd [M] are written unless both are NULL.  y may be x. */
int32_t nf_layernorm_fwd(const nf_layernorm_desc *d, int64_t M, const void *x, const float *gamma, const float *beta,
                         void *y, float *mean, float *rstd, void *stream);
/* With xh = (x - mean) rstd and g = dy gamma: dx = rstd (g - avg(g) - xh avg(g xh)) + dr, averages over the row; dgamma = sum dy xh,
 * dbeta = sum dy over the rows.  mean and rstd are what the forward wrote.  gamma may be NULL (1), dr too (a residual path's
 * gradient, read in the same pass; dx may be dy or dr).  Any of dx, dgamma, dbeta may be NULL, not all; ws is wanted where dgamma or dbeta is given. */
int32_t nf_layernorm_bwd(const nf_layernorm_desc *d, int64_t M, const void *dy, const void *x, const float *gamma,
                         const float *mean, const float *rstd, const void *dr, void *dx, float *dgamma, float *dbeta,
                         void *ws, size_t ws_bytes, void *stream);

/* The activation cache in 8 or 4 bits an element.  A row of n elements is cut into groups of 32 (the last may be
 * shorter); group j has the exponent byte scales[row][j] = E + 127 and its elements are code * 2^E:
 *   NF_Q_INT8  signed bytes -127 ... 127
 *   NF_Q_E4M3  8-bit floats, 4 exponent bits, largest 448
 *   NF_Q_E2M1  4-bit floats 0, .5, 1, 1.5, 2, 3, 4, 6 with a sign, two to a byte, the earlier element in the low half
 * E is the least (>= -127) with which the group's largest magnitude is at most the largest code; codes are rounded to
 * nearest, ties to even (next to the largest fp32 number that may be an infinity).  A group that holds an infinity or a NaN gets the exponent byte 255 and reads back as NaN.
 * Row strides are nf_qcache_row_bytes: the codes' bytes and the exponents' bytes, both rounded up to 16.
 * Write stores batch rows at [first, first+B); read gathers as nf_cache_read does (an index outside [0, capacity)
 * is clamped).  Labels as there. */
enum { NF_Q_INT8 = 0, NF_Q_E4M3 = 1, NF_Q_E2M1 = 2 };
int32_t nf_qcache_row_bytes(int32_t format, int64_t n, size_t *code_bytes, size_t *scale_bytes);
int32_t nf_qcache_write(int32_t format, int32_t dtype, uint8_t *codes, uint8_t *scales, int32_t *cache_labels,
                        int64_t capacity, int64_t n, int64_t first, int32_t B, const void *x, const int32_t *labels,
                        void *stream);
int32_t nf_qcache_read(int32_t format, int32_t dtype, const uint8_t *codes, const uint8_t *scales,
                       const int32_t *cache_labels, int64_t capacity, int64_t n, int64_t first, const int64_t *idx,
                       int32_t B, void *x_out, int32_t *labels_out, void *stream);

/* Matrices in 4 bits, and their products.  A matrix [rows][cols] is held as the rows of an NF_Q_E2M1 cache of n = cols (the same codes, exponents and
 * row strides: nf_qcache_row_bytes; nf_qcache_write fills and nf_qcache_read reads one, too).  nf_mx_quantise writes x [rows][cols], of
 * type dtype, by rows into codes and scales, and by columns, that is as the matrix [cols][rows], into codes_t and scales_t; either pair may be
 * NULL.  Codes behind a row's last element, up to a whole group, are 0; other bytes between a row's end and its stride are left as they
 * are, and products read none of them as numbers.  Beyond 2^32 groups by rows, 2^24 tiles of 128 x 64 by columns or
 * 2^44 elements: NF_ERR_UNSUPPORTED. */
int32_t nf_mx_quantise(int32_t dtype, int64_t rows, int64_t cols, const void *x, uint8_t *codes, uint8_t *scales,
                       uint8_t *codes_t, uint8_t *scales_t, void *stream);
/* y = r + act(a b^T + bias) [M][N]: a holds M rows of K, b N rows of K, both in 4 bits; d->dtype is that of y and r; bias and r may be
 * NULL.  Sums are fp32 (a group that reads back as NaN makes its results NaN).  A linear layer's gradients are such products, each operand
 * quantised along the axis that is summed over: dx = product(dz by rows, W by columns), dW = product(dz by columns, x by columns).
 * 1 <= M < 2^31 - 512, N <= 2^20, K <= 2^24, and the tiles of 64 along M times those along N stay below 2^23. */
int32_t nf_mx_product_workspace_bytes(const nf_linear_desc *d, int64_t M, size_t *out);
int32_t nf_mx_product(const nf_linear_desc *d, int64_t M, const uint8_t *a, const uint8_t *a_scales, const uint8_t *b,
                      const uint8_t *b_scales, const float *bias, const void *r, void *y, void *ws, size_t ws_bytes,
                      void *stream);
/* nf_linear_fwd with W [N][K] in 4 bits: x [M][K], of type dtype, is quantised by rows on the way (up to 32 rows within the product's
 * launch, else into the workspace).  b, r, drop, z as there.  The results are those of nf_mx_quantise and nf_mx_product. */
int32_t nf_mx_linear_workspace_bytes(const nf_linear_desc *d, int64_t M, size_t *out);
int32_t nf_mx_linear_fwd(const nf_linear_desc *d, int64_t M, const void *x, const uint8_t *W, const uint8_t *W_scales,
                         const float *b, const void *r, const nf_dropout_desc *drop, void *y, void *z, void *ws,
                         size_t ws_bytes, void *stream);

/* ---- Profiler and Partitioner ("Modules", Algorithm 1): host functions, no device work ---------
 * The Profiler's measured memory is replaced by the exact device bytes of one local step with
 * this library: parameters + gradients (+ momentum buffers) of the layer and its head, the input,
 * shortcut and emitted batches, labels, and nf_workspace_bytes.  nf_fit_linear is the Profiler's
 * linear model (least squares: bytes ~ intercept + slope * batch); nf_profile_layer evaluates the
 * byte count at n (2..64) batch sizes and fits it.  nf_partition is Algorithm 1: per layer the
 * largest batch size whose model stays within the budget M (same unit as the models), capped at
 * B_limit; then consecutive layers are grouped into one block while
 * |b[i+1] - b[i]| <= rho * b[i], a block taking the smallest batch size of its layers.
 * Outputs: layer_batch[n_layers] (optional), block_first[k] = index of the first layer of block
 * k and block_batch[k] (arrays of n_layers entries), *n_blocks.  A layer that does not fit at
 * batch size 1 gets batch size 0. */
typedef struct {
  double slope, intercept;
} nf_linear_model;
int32_t nf_layer_step_bytes(const nf_layer_desc *d, const nf_aux_desc *a, int32_t B, int32_t with_momentum,
                            size_t *out);
int32_t nf_fit_linear(int32_t n, const double *batch, const double *bytes, nf_linear_model *out);
int32_t nf_profile_layer(const nf_layer_desc *d, const nf_aux_desc *a, int32_t with_momentum, int32_t n,
                         const int32_t *batches, nf_linear_model *out);
int32_t nf_partition(int32_t n_layers, const nf_linear_model *R, double M, int32_t B_limit, double rho,
                     int32_t *layer_batch, int32_t *block_first, int32_t *block_batch, int32_t *n_blocks);

/* ---- measurement aid (not a step of the method) ---------------------------------------------
 * Between nf_prof_begin and nf_prof_end every kernel the library enqueues is bracketed by a
 * HIP-event pair on the caller's stream.  nf_prof_end waits for those events (the only call
 * that blocks the host), and returns one record per kernel: launches, summed duration (ms),
 * summed algorithmic FLOPs and bytes.  Records are sorted by duration, at most `cap` are
 * written, *n receives the number of distinct kernels.  Kernels that a call puts into one launch (the two
 * weight gradients of small steps, both gradients of a linear layer) are launched and recorded one by one after nf_prof_begin;
 * nf_prof_begin_as_run records the launches that a call makes without a measurement, such a one under
 * a name of its own.  Process-wide state (one recording at a time;
 * the record list is guarded by a mutex so that launches from several host threads may be recorded),
 * creates HIP events: keep it out of production loops. */
typedef struct {
  char kernel[48];
  int64_t launches;
  double ms, flops, bytes;
} nf_prof_record;
/* Compute units and peak shader clock (kHz) of the current device, as the runtime reports them
 * (the fp32 MFMA peak is compute_units x 4 SIMDs x 64 flop/clk x clock). */
int32_t nf_device_info(int32_t *compute_units, int32_t *clock_khz);
int32_t nf_prof_begin(void);
int32_t nf_prof_begin_as_run(void);
int32_t nf_prof_end(nf_prof_record *out, int32_t cap, int32_t *n);

#ifdef __cplusplus
}
#endif
#endif
