/*
 * imbd.h -- C ABI of the MI355X (gfx950) hot path of integrated model/batch/domain
 * parallel SGD (Gholami, Azad, Jin, Keutzer, Buluc, arXiv:1712.04432).
 *
 * One process's share of the P_r x P_c grid: for each fully connected layer the three
 * products Y = W X, Delta_W = Delta_Y X^T and Delta_X = W^T Delta_Y (Sec. 1; Appendix A),
 * the nonlinearity and its derivative, softmax cross-entropy at the top and the
 * mini-batch SGD update of Eq. (1). Also a 3x3 convolution tile of a domain-parallel
 * layer with its halo supplied (Sec. 2.2).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Memory. Every tensor pointer is a DEVICE pointer owned by the caller; the library
 *   never frees or keeps it. Calls enqueue work on `stream` (a hipStream_t passed as
 *   void*, NULL = the default stream) and return without synchronising. No call
 *   allocates device memory: scratch space comes in through a `ws` argument sized by the
 *   matching *_workspace_bytes function.
 * - Layout. The paper stores one sample per column (X_i is d_{i-1} x B); here one sample
 *   is one row of a row-major array, X[b][k], which is the same bytes as the paper's
 *   column-major X_i. Weights W_i are row-major [d_i][d_{i-1}] as in the paper.
 *   "ld" arguments are leading dimensions in ELEMENTS (>= the row length), so process
 *   blocks of a larger array are passed as views without copies.
 * - Types. IMBD_BF16 operands are bfloat16 bit patterns (uint16). Accumulation is
 *   always fp32; master weights, biases, gradients and the loss are fp32.
 *   Conversions to bf16 round to nearest, ties to even.
 * - Errors. Arguments are validated on the host before anything is enqueued; a bad
 *   argument returns IMBD_EINVAL and enqueues nothing. A launch failure returns IMBD_EHIP.
 *   imbd_last_error() gives a thread-local description of the last failure. No C++
 *   exception crosses this boundary. Labels outside [0, C) are not read out of bounds;
 *   their sample's loss and its whole row of the top-layer gradient become NaN, so the
 *   batch loss and every update computed from that gradient are NaN too.
 * - Determinism. Fixed reduction orders: identical inputs give identical bits.
 * - Concurrency. Calls that share a workspace must be ordered on one stream.
 */
#ifndef IMBD_H
#define IMBD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum imbd_status {
    IMBD_OK = 0,
    IMBD_EINVAL = -1,       /* bad argument (null pointer, size, leading dimension, enum) */
    IMBD_EUNSUPPORTED = -2, /* valid request the library has no kernel for */
    IMBD_EHIP = -3,         /* the HIP runtime reported an error */
    IMBD_EWORKSPACE = -4    /* workspace missing or smaller than *_workspace_bytes says */
};

enum imbd_dtype { IMBD_F32 = 0, IMBD_BF16 = 1 };

/* Static description of a status code; never NULL. mlp_status_string is the same
 * function under the name the rest of the mlp_* calls use. */
const char *imbd_status_string(int status);
const char *mlp_status_string(int status);
/* Detail of the last failure on the calling thread ("" if none). */
const char *imbd_last_error(void);
/* Library version, major*10000 + minor*100 + patch. */
int imbd_version(void);

/* ====================================================================================
 * Whole network (one process holding the full W_i and a batch of B samples: the
 * P_r = P_c = 1 case of Sec. 2.3)
 * ==================================================================================== */

/* A network of L fully connected layers d_0 -> d_1 -> ... -> d_L: ReLU after every
 * hidden layer, softmax cross-entropy on the top layer's logits. */
typedef struct {
    int n_layers;      /* L >= 1 */
    const int *dims;   /* HOST array of L+1 widths d_0..d_L, each >= 1 */
    int batch;         /* B >= 1 */
    int dtype;         /* IMBD_F32 or IMBD_BF16: type of weights copies and activations */
} imbd_mlp_desc;

/* Parameters of layer i (all device pointers, caller-owned). */
typedef struct {
    float *w;      /* fp32 master weights [d_i][d_{i-1}], contiguous */
    void *w_lp;    /* IMBD_BF16: bf16 copy [d_i][d_{i-1}] read by the products; IMBD_F32: == w */
    float *b;      /* fp32 bias [d_i] */
    float *dw;     /* fp32 [d_i][d_{i-1}]: Delta_W output when the update is not fused, else unused */
    float *db;     /* fp32 [d_i]: bias gradient output when the update is not fused, else unused */
} imbd_layer;

/* Bytes of workspace mlp_fwd/mlp_bwd need for this network (0 if the desc is invalid).
 * It holds X_2..X_L, the logits, every Delta_Y_i, the per-sample losses and the
 * split-K partial sums. */
size_t mlp_workspace_bytes(const imbd_mlp_desc *desc);

enum imbd_ws_kind {
    IMBD_WS_ACT = 0,     /* X_{i+1} = f(Y_i) for layer i in 1..L-1, [B][d_i] in desc->dtype */
    IMBD_WS_LOGITS = 1,  /* Y_L, [B][d_L] fp32 (layer argument ignored) */
    IMBD_WS_DY = 2,      /* Delta_Y_i for layer i in 1..L, [B][d_i] in desc->dtype */
    IMBD_WS_ROWLOSS = 3  /* per-sample loss, [B] fp32 (layer argument ignored) */
};
/* Byte offset of a region inside the workspace, or -1 for an invalid request. */
int64_t mlp_workspace_offset(const imbd_mlp_desc *desc, int kind, int layer);

/* Forward pass and loss (Sec. 1: Y_i = W_i X_i + b_i, X_{i+1} = f(Y_i); softmax
 * cross-entropy at the top). x: [B][d_0] input batch in desc->dtype. labels: [B] int32
 * class indices in [0, d_L). loss: device fp32 scalar, the batch-mean loss. Also leaves
 * Delta_Y_L = (softmax - onehot)/B in the workspace for mlp_bwd: the 1/B of Eq. (1) is
 * applied here, once. */
int mlp_fwd(const imbd_mlp_desc *desc, const imbd_layer *layers, const void *x,
            const int32_t *labels, void *ws, size_t ws_bytes, float *loss, void *stream);

/* Backward pass (Sec. 1 and Appendix A.2): for i = L..1, Delta_W_i = Delta_Y_i X_i^T,
 * db_i = Delta_Y_i 1, and for i >= 2 Delta_Y_{i-1} = (W_i^T Delta_Y_i) * [X_i > 0].
 * Needs the workspace of the mlp_fwd call just before it (same desc, same x).
 * fuse_sgd != 0: apply Eq. (1) in the weight-gradient epilogue,
 *   w <- w - lr*Delta_W, w_lp <- bf16(w), b <- b - lr*db, without storing Delta_W;
 *   each layer's Delta_X product is issued before its update, so it reads the old W.
 * fuse_sgd == 0: store Delta_W into layers[i].dw and db into layers[i].db; no update.
 * dx1: optional [B][d_0] output in desc->dtype for Delta_X_1 = W_1^T Delta_Y_1 (not
 * needed for training: the backward sum of Sec. 2.2 starts at layer 2); NULL skips it. */
int mlp_bwd(const imbd_mlp_desc *desc, imbd_layer *layers, const void *x, void *ws,
            size_t ws_bytes, int fuse_sgd, float lr, void *dx1, void *stream);

/* One SGD iteration: mlp_fwd followed by mlp_bwd with the update fused. */
int mlp_train_step(const imbd_mlp_desc *desc, imbd_layer *layers, const void *x,
                   const int32_t *labels, void *ws, size_t ws_bytes, float lr, float *loss,
                   void *stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): mlp_train_step with its workspace
 * taken from a scratch array inside the library instead of a ws argument. The array
 * holds IMBD_STATIC_SCRATCH_BYTES on every GPU the library runs on, from the library's
 * load until the process ends; the call itself allocates nothing. The caller still
 * passes parameters, input, labels and the loss. Results are those of mlp_train_step.
 * Returns IMBD_EWORKSPACE, enqueueing nothing, when mlp_workspace_bytes(desc) exceeds
 * the scratch (the 9216-4096-4096-1000 stack at B = 256 needs 46 MiB, 25088-4096-4096-1000
 * at B = 512 needs 53 MiB). All calls on one GPU share that GPU's one array, which keeps
 * the last call's contents: calls that overlap on one GPU (other streams, other threads)
 * race, so order them on one stream. The current device must be the stream's device. */
#define IMBD_STATIC_SCRATCH_BYTES (64u << 20)
int mlp_train_step_static(const imbd_mlp_desc *desc, imbd_layer *layers, const void *x,
                          const int32_t *labels, float lr, float *loss, void *stream);

/* ====================================================================================
 * Update and conversion
 * ==================================================================================== */

/* Eq. (1) on n parameters: w <- w - lr * grad_scale * grad (fp32, one rounding), then,
 * if w_lp != NULL and lp_dtype == IMBD_BF16, w_lp <- bf16(w). grad_scale = 1 when the
 * gradient already is the mini-batch mean. n == 0 is a no-op. Used for biases and for
 * local blocks after an external reduction. */
int sgd_step(float *w, void *w_lp, int lp_dtype, const float *grad, int64_t n, float lr,
             float grad_scale, void *stream);

/* dst[i] = bf16(src[i]) (round to nearest even; NaN stays NaN), n >= 0. */
int cast_f32_bf16(const float *src, uint16_t *dst, int64_t n, void *stream);

/* ====================================================================================
 * Single operations (the top of the network and single-layer products)
 * ==================================================================================== */

/* Softmax cross-entropy over C classes for B samples (the loss of Sec. 1 and App. A.2):
 * logits [B][ldz] fp32; loss = inv_batch * sum_b (logsumexp_c z_b - z_b[label_b]);
 * dz [B][lddz] in dz_dtype = inv_batch * (softmax(z_b) - onehot(label_b)).
 * row_loss: device fp32 [B] scratch that also receives the per-sample losses.
 * dz may be NULL (loss only). */
int softmax_xent(int B, int C, const float *logits, int64_t ldz, const int32_t *labels,
                 float inv_batch, float *loss, float *row_loss, void *dz, int64_t lddz,
                 int dz_dtype, void *stream);

/* ====================================================================================
 * Local blocks of one process (r, c) of the P_r x P_c grid (Sec. 2.3, the 1.5D
 * algorithm; Appendix A). The process holds a (d_i/P_r) x d_{i-1} row block of W_i and a
 * column block of B/P_c samples of X_i and Y_i. Outputs are left UNREDUCED: Y_blk waits
 * for the all-gather over P_r, the Delta_W partial for the all-reduce over P_c and the
 * Delta_X partial for the all-reduce over P_r (those collectives are not part of this
 * library). P_r, P_c >= 1 describe the grid; d_out_blk = d_i/P_r and b_blk = B/P_c are
 * the local sizes.
 * ==================================================================================== */

/* Y_blk = W_blk X_blk + b_blk (App. A.1, model-parallel form on the local samples),
 * then ReLU if relu != 0.
 * w_blk [d_out_blk][ldw] and x_blk [b_blk][ldx] in dtype; b_blk_bias [d_out_blk] fp32 or
 * NULL; y_blk [b_blk][ldy] in y_dtype (IMBD_F32 for logits).
 * ws/ws_bytes: scratch for split-K partial sums, see mlp_local_workspace_bytes. */
int mlp_local_fwd(int dtype, int relu, int P_r, int P_c, int d_out_blk, int d_in, int b_blk,
                  const void *w_blk, int64_t ldw, const float *b_blk_bias,
                  const void *x_blk, int64_t ldx, void *y_blk, int64_t ldy, int y_dtype,
                  void *ws, size_t ws_bytes, void *stream);

/* Backward products of the block (App. A.2):
 *   dw_part[m][k] = (1/B) sum_{b in block} dy_blk[b][m] x_blk[b][k],   B = b_blk * P_c
 *   db_part[m]    = (1/B) sum_{b in block} dy_blk[b][m]
 *   dx_part[b][k] = sum_m w_blk[m][k] dy_blk[b][m]  (times [x_blk[b][k] > 0] if mask_relu)
 * dy_blk is the raw per-sample gradient dJ/dY for J = sum_b f_b; the 1/B of Eq. (1) is
 * the global batch's, so the P_c partials sum to the mini-batch mean gradient. The
 * ReLU mask uses this layer's input block, which is the same on every process of the
 * grid column, so it commutes with the all-reduce over P_r.
 * w_blk [d_out_blk][ldw], x_blk [b_blk][ldx], dy_blk [b_blk][lddy] in dtype;
 * dw_part [d_out_blk][lddw] fp32; db_part [d_out_blk] fp32 or NULL;
 * dx_part [b_blk][lddx] fp32 or NULL (skip). b_blk == 0 writes zero partials. */
int mlp_local_bwd(int dtype, int P_r, int P_c, int d_out_blk, int d_in, int b_blk,
                  const void *w_blk, int64_t ldw, const void *dy_blk, int64_t lddy,
                  const void *x_blk, int64_t ldx, float *dw_part, int64_t lddw, float *db_part,
                  float *dx_part, int64_t lddx, int mask_relu, void *ws, size_t ws_bytes,
                  void *stream);

/* Workspace bytes for mlp_local_fwd (which = 0) or mlp_local_bwd (which = 1) at these
 * sizes. */
size_t mlp_local_workspace_bytes(int which, int dtype, int d_out_blk, int d_in, int b_blk);

/* ====================================================================================
 * A fully connected layer of any network: the product of Sec. 1 with an activation of choice and
 * a residual in its epilogue, and the products of its backward pass with the derivative of
 * the activation below and the residual's gradient in theirs. Layouts as for the local blocks: w
 * [d_out][ldw], x [B][ldx] in dtype, one sample per row; any strides, any alignment.
 * Sizes (IMBD_EUNSUPPORTED past them): widths up to 2^30, fewer than 2^31 - 1024 samples, and no launch of 2^24
 * workgroups or more. No output may overlap an input or another output, but for a residual in the
 * place of the output that it is added to (same address, leading dimension and type).
 * ==================================================================================== */
enum imbd_act {
    IMBD_ACT_NONE = 0,      /* v */
    IMBD_ACT_RELU = 1,      /* max(v, 0); derivative 1 where v > 0 */
    IMBD_ACT_GELU = 2,      /* v Phi(v), Phi the standard normal distribution */
    IMBD_ACT_GELU_TANH = 3, /* v (1 + tanh(sqrt(2/pi) (v + 0.044715 v^3))) / 2 */
    IMBD_ACT_SILU = 4       /* v / (1 + e^-v) */
};

/* Workspace bytes for linear_fwd (which = 0) or linear_bwd (which = 1) at these sizes: 0 for
 * sizes that they refuse, and maybe for others (then ws is not read). ws is 256-byte aligned. */
size_t linear_workspace_bytes(int which, int dtype, int d_out, int d_in, int B);

/* z = W x + bias,  y = act(z) + residual. bias [d_out] fp32 or NULL; residual [B][ldr] in y_dtype or
 * NULL; y [B][ldy] in y_dtype; z [B][ldz] in dtype, or NULL: not kept (linear_bwd of the layer above
 * needs it unless act is none). Sums, act and residual in fp32, y and z rounded once each (y
 * does not see z's rounding). */
int linear_fwd(int dtype, int act, int d_out, int d_in, int B, const void *w, int64_t ldw,
               const float *bias, const void *x, int64_t ldx, const void *residual, int64_t ldr,
               void *y, int64_t ldy, int y_dtype, void *z, int64_t ldz, void *ws, size_t ws_bytes,
               void *stream);

/* The backward products, each skipped where its output is NULL (not all three). dy [B][lddy] in
 * dtype is the gradient before this layer's own activation, at W x + bias:
 *   dx = (W^T dy) * act'(z) + residual     x = act(z) is the output of the layer below
 *   dw[o][i] = sum_b dy[b][o] x[b][i]      db[o] = sum_b dy[b][o]
 * so that dx is the dy of the layer below (or, with act none, the gradient of x itself). z [B][ldz]
 * in dtype, not read where act is none; residual [B][ldr] in dx_dtype or NULL: what else flows back
 * to the same place; dx [B][lddx] in dx_dtype; dw [d_out][lddw] and db [d_out] fp32. w may be NULL
 * without dx, x without dw. B == 0 writes zeros to dw and db. */
int linear_bwd(int dtype, int act, int d_out, int d_in, int B, const void *w, int64_t ldw,
               const void *dy, int64_t lddy, const void *x, int64_t ldx, float *dw, int64_t lddw,
               float *db, const void *z, int64_t ldz, const void *residual, int64_t ldr, void *dx,
               int64_t lddx, int dx_dtype, void *ws, size_t ws_bytes, void *stream);

/* dz = dy * act'(z), d columns, all in dtype: for a layer whose own activation is followed by a residual, dy the
 * gradient of its y. (A residual itself receives dy.) dz may be dy or z (same leading dimension). */
int act_bwd(int dtype, int act, int B, int d, const void *dy, int64_t lddy, const void *z, int64_t ldz,
            void *dz, int64_t lddz, void *stream);

/* ====================================================================================
 * Domain-parallel 3x3 convolution tile (Sec. 2.2, Fig. of the domain split; sizes from
 * Eq. (2)). Stride 1, "same" padding, cross-correlation, channels-last bf16 operands:
 *   x_pad  [N][H+2][W+2][C_in]  : the tile plus its 1-pixel halo (zeros on the image border)
 *   w      [C_out][3][3][C_in]
 *   dy_pad [N][H+2][W+2][C_out] : output gradient with its 1-pixel halo from the
 *                                 neighbouring tiles (output-side halo term of Eq. (7))
 * ==================================================================================== */

/* y[n][h][w][o] = sum_{r,s,c} w[o][r][s][c] x_pad[n][h+r][w+s][c]; y [N][H][W][C_out] in
 * y_dtype. */
int conv3x3_tile_fwd(int N, int H, int W, int C_in, int C_out, const void *x_pad,
                     const void *w, void *y, int y_dtype, void *stream);

/* dx[n][h][w][c] = sum_{r,s,o} w[o][r][s][c] dy_pad[n][h+2-r][w+2-s][o];
 * dx [N][H][W][C_in] in dx_dtype. */
int conv3x3_tile_dgrad(int N, int H, int W, int C_in, int C_out, const void *dy_pad,
                       const void *w, void *dx, int dx_dtype, void *stream);

/* The tile's partial weight gradient (the all-reduce over all processes of Eq. (7)
 * completes it): dw[o][r][s][c] = sum_{n,h,w} dy[n][h][w][o] x_pad[n][h+r][w+s][c],
 * dy = interior of dy_pad; dw [C_out][3][3][C_in] fp32. ws (16-byte aligned) holds the partial
 * sums of ranges of the positions. conv3x3_wgrad_workspace_bytes is the size to bring: from it
 * on, the ranges, and so the order of the sums and dw's bits, are the same. Some shapes accept
 * less, down to none (IMBD_EWORKSPACE below the least): dw is then summed over fewer ranges,
 * more slowly and in another order. */
int conv3x3_tile_wgrad(int N, int H, int W, int C_in, int C_out, const void *x_pad,
                       const void *dy_pad, float *dw, void *ws, size_t ws_bytes, void *stream);
size_t conv3x3_wgrad_workspace_bytes(int N, int H, int W, int C_in, int C_out);

/* The tile's whole backward pass (Sec. 2.2; Eq. (7) for what it exchanges): the input
 * gradient (as conv3x3_tile_dgrad, skipped when dx is NULL) and the partial weight
 * gradient (as conv3x3_tile_wgrad), on `stream` in that order. Both passes are validated
 * before either is enqueued; ws as for conv3x3_tile_wgrad. */
int conv3x3_tile_bwd(int N, int H, int W, int C_in, int C_out, const void *x_pad, const void *w,
                     const void *dy_pad, void *dx, int dx_dtype, float *dw, void *ws,
                     size_t ws_bytes, void *stream);

/* ====================================================================================
 * A fully connected layer whose weights are split into E experts: every sample (token)
 * goes through the k experts that its router prefers, and its k results are summed with
 * their gates. One process's share, as above: w [E][d_out][ldw] holds one W_i per expert.
 *
 * The (token, expert) pairs are kept in EXPERT ORDER: pair by pair in the order of (expert,
 * token, choice), each at its SLOT 0 .. offsets[E] - 1; expert e owns the slots
 * offsets[e] .. offsets[e+1] - 1 (none, one or all of them). offsets, rows and slots are
 * DEVICE int32 arrays, so no call waits for the GPU. Their values are not trusted: offsets
 * are clamped to [0, n_rows] (an expert whose end lies before its start has no slots), and an
 * index outside its array reads as zeros and writes nothing. One slot belongs to one expert
 * and to one (token, choice): where offsets overlap or slots name a slot twice, the outputs
 * there are undefined.
 * Sizes (IMBD_EUNSUPPORTED past them): 1 <= E <= 512 and 1 <= k <= 16; fewer than 2^31 - 1024
 * slots, rows and tokens; widths up to 2^30; and no launch of 2^24 workgroups or more: a tile of
 * rows, 4 tokens (expert_combine_bwd), 4 to 32 tokens (expert_route_bwd). No output may overlap an input or another output.
 * ==================================================================================== */

/* The router. logits [T][ldl] fp32, ldl >= E. Each token's k largest logits, in descending
 * order, ties to the lowest expert: experts [T][k], and
 *   gates[t][j] = exp(z_e) / sum exp(z)   over all E experts, or with renorm != 0 over the k
 *                                         chosen ones.
 * An expert whose logit is -inf is never chosen: where fewer than k are left (a padding
 * token's row of -inf: none), experts[t][j] = -1, gates[t][j] = 0 and slots[t][j] = -1, and
 * the pair has no slot. A NaN logit counts as the largest; it or +inf makes the row's gates
 * NaN. Also the plan in expert order: offsets [E+1], rows [T*k] (the token of each slot;
 * entries from offsets[E] on are left as they were) and slots [T][k] (each pair's slot).
 * All outputs contiguous. T == 0 writes zeros to offsets only.
 * ws (256-byte aligned): expert_route_workspace_bytes(T, E, k), which is 0 for sizes that
 * expert_route refuses and may be 0 for others too (then ws is not read). */
size_t expert_route_workspace_bytes(int T, int E, int k);
int expert_route(int T, int E, int k, int renorm, const float *logits, int64_t ldl, float *gates,
                 int32_t *experts, int32_t *offsets, int32_t *rows, int32_t *slots, void *ws,
                 size_t ws_bytes, void *stream);

/* The logits' gradient from the gates': dgates [T][k] contiguous, dlogits [T][lddl] fp32 (all E
 * of a row are written). gates and experts as expert_route left them, logits the same input
 * (read for renorm == 0 only, else it may be NULL). With p the softmax over all E,
 *   renorm:  dz_e = sum_j [experts_j = e] g_j (dg_j - sum_i g_i dg_i)
 *   else:    dz_e = sum_j [experts_j = e] g_j dg_j - p_e sum_i g_i dg_i
 * A pair with experts[t][j] = -1 counts for nothing. */
int expert_route_bwd(int T, int E, int k, int renorm, const float *logits, int64_t ldl,
                     const float *gates, const int32_t *experts, const float *dgates,
                     float *dlogits, int64_t lddl, void *stream);

/* Every expert's forward product on its slots, y[s] = W_e x[rows[s]] + b_e, then ReLU if
 * relu != 0, for the slots s of expert e. rows NULL: x is in expert order already (x[s],
 * n_x == n_rows). n_rows: the number of rows of y (and of `rows`), at least offsets[E] if the
 * offsets are to be served whole; rows of y that no expert owns are left as they were. n_x:
 * the number of rows of x; a slot whose rows[s] is outside [0, n_x) reads a row of zeros.
 * w: expert e's matrix at w + e*sw, [d_out][ldw], in dtype (sw >= (d_out-1)*ldw + d_in unless
 * E == 1); bias [E][d_out] fp32 contiguous or NULL; x [n_x][ldx] in dtype; y [n_rows][ldy] in
 * y_dtype. Sums in fp32, one rounding to y_dtype after bias and ReLU. */
int expert_fwd(int dtype, int relu, int E, int d_out, int d_in, int n_rows, int n_x, const void *w,
               int64_t ldw, int64_t sw, const float *bias, const void *x, int64_t ldx,
               const int32_t *rows, const int32_t *offsets, void *y, int64_t ldy, int y_dtype,
               void *stream);

/* Their backward products, each skipped where its output is NULL (not all three):
 *   dx[s]      = W_e^T dy[s]  (times [x[rows[s]] > 0] if mask_relu)   in expert order
 *   dw_e[o][i] = sum over e's slots s of dy[s][o] x[rows[s]][i]
 *   db_e[o]    = sum over e's slots s of dy[s][o]
 * No factor 1/B: dy carries it. dy [n_rows][lddy] in dtype; x, rows, n_x, w as for expert_fwd
 * (x may be NULL where neither dw nor mask_relu needs it, w where dx is NULL); dw expert by
 * expert at dw + e*sdw, [d_out][lddw] fp32; db [E][d_out] fp32 contiguous; dx [n_rows][lddx] in
 * dx_dtype. dw and db of an expert without slots are zero; rows of dx that no expert owns are
 * left as they were. The gradient of x[t] itself is the sum of its slots' rows of dx:
 * expert_combine with gates NULL. */
int expert_bwd(int dtype, int E, int d_out, int d_in, int n_rows, int n_x, const void *w, int64_t ldw,
               int64_t sw, const void *dy, int64_t lddy, const void *x, int64_t ldx,
               const int32_t *rows, const int32_t *offsets, float *dw, int64_t lddw, int64_t sdw,
               float *db, void *dx, int64_t lddx, int dx_dtype, int mask_relu, void *stream);

/* Back to token order: y[t] = sum_j gates[t][j] ys[slots[t][j]] (gates NULL: 1), summed in fp32
 * in the order of j. ys [n_rows][ldys] in dtype, y [T][ldy] in y_dtype, d columns; slots [T][k]
 * and gates [T][k] contiguous; a slot outside [0, n_rows) adds nothing (whatever its gate). */
int expert_combine(int dtype, int T, int k, int d, int n_rows, const void *ys, int64_t ldys,
                   const int32_t *slots, const float *gates, void *y, int64_t ldy, int y_dtype,
                   void *stream);

/* Its backward pass: dys[slots[t][j]] = gates[t][j] dy[t] and dgates[t][j] = dy[t] . ys[slots[t][j]]
 * (0 for a slot outside [0, n_rows)). dy [T][lddy], ys [n_rows][ldys] and dys [n_rows][lddys] in
 * dtype; rows of dys that no slot names are left as they were. dgates [T][k] or NULL (then ys is
 * not read). dys may not overlap ys. */
int expert_combine_bwd(int dtype, int T, int k, int d, int n_rows, const void *dy, int64_t lddy,
                       const void *ys, int64_t ldys, const int32_t *slots, const float *gates,
                       void *dys, int64_t lddys, float *dgates, void *stream);

/* ====================================================================================
 * What a vocabulary's logits are for, beside softmax_xent: distillation from a teacher, and
 * the log probabilities of given tokens. B rows (tokens) of V logits, fp32 or bf16, [B][ldz].
 *
 * With q the softmax of z / temperature over all V. A logit of -inf rules its token out (q = 0); a
 * NaN or +inf makes its row's results NaN, as does a row of -inf only (its lse is -inf). Statistics and sums in
 * fp32, in a fixed order. Sizes (IMBD_EUNSUPPORTED past them): B < 2^24, V <= 2^30, K <= 256, n <= 64.
 * ws (256-byte aligned): the *_workspace_bytes function's, which is 0 for sizes that the call refuses
 * and may be 0 for others too (then ws is not read). No output may overlap an input or another output,
 * but dlogits may be logits itself (same address, leading dimension and type), which then holds
 * the gradient instead.
 * ==================================================================================== */

/* Divergence of the student's softmax q from a teacher's, of whose logits K are known in each
 * row: ids [B][K] their tokens, teacher [B][K] fp32 their values t, both contiguous, in any order.
 *   p_j = exp(t_j / temperature) / sum over the row's K, or with lse != NULL (fp32 [B], the logsumexp
 *         of all the teacher's logits / temperature)  exp(t_j / temperature - lse[b])
 *   row_loss[b] = w_b temperature^2 sum_j p_j (log p_j - log q_{id_j})
 *   loss        = inv_batch sum_b row_loss[b]
 *   dlogits[b][v] = inv_batch w_b temperature (q_v sum_j p_j - sum_j [id_j = v] p_j)
 * w = weight (fp32 [B], NULL: 1). An entry with id < 0 or t = -inf is no entry (rows with fewer than
 * K); the same id twice counts as the sum of both. A row without entries or with w_b = 0 has
 * row_loss 0 and a gradient of zeros, whatever its logits hold; one with an id >= V (and w_b != 0)
 * has NaN in both, and so has the loss. dlogits [B][lddl] in dlogits_dtype, or NULL (loss only). */
size_t distill_workspace_bytes(int B, int V, int K);
int distill_xent(int dtype, int B, int V, int K, const void *logits, int64_t ldz, const int32_t *ids,
                 const float *teacher, const float *lse, const float *weight, float temperature,
                 float inv_batch, float *loss, float *row_loss, void *dlogits, int64_t lddl,
                 int dlogits_dtype, void *ws, size_t ws_bytes, void *stream);

/* Of every row: logp [B] = log q_{tokens[b]}, and where they are not NULL entropy [B] = -sum q log q,
 * lse [B] = log sum exp(z / temperature), and the n largest logits in descending order, ties to the lowest token:
 * top_ids [B][n] and top_logp [B][n] = log q of them (n == 0: neither). tokens[b] < 0: no
 * token, logp 0; tokens[b] >= V: logp NaN. Alternatives are chosen by the logits themselves; a token
 * that is ruled out or whose logit is NaN is none: where fewer than n are left, id -1 and log
 * probability -inf. All fp32 or int32, contiguous. */
size_t token_logprobs_workspace_bytes(int B, int V, int n);
int token_logprobs(int dtype, int B, int V, int n, const void *logits, int64_t ldz, const int32_t *tokens,
                   float temperature, float *logp, float *entropy, float *lse, int32_t *top_ids,
                   float *top_logp, void *ws, size_t ws_bytes, void *stream);

/* The logits' gradient from dlogp [B] and dentropy [B] (either may be NULL: zeros), with lse and entropy
 * as token_logprobs left them for the same logits, tokens and temperature (entropy may be NULL without dentropy):
 *   dlogits[b][v] = (g_b ([v = tokens[b]] - q_v) - h_b q_v (log q_v + entropy[b])) / temperature
 * (log q_v is taken from lse, so it is as exact as an fp32 lse is: off by 2^-23 |lse|.)
 * g_b = dlogp[b], 0 where tokens[b] < 0 (tokens[b] >= V: the row becomes NaN); h = dentropy. A row
 * with g_b = h_b = 0 becomes zeros, whatever its logits hold. */
int token_logprobs_bwd(int dtype, int B, int V, const void *logits, int64_t ldz, const int32_t *tokens,
                       float temperature, const float *lse, const float *entropy, const float *dlogp,
                       const float *dentropy, void *dlogits, int64_t lddl, int dlogits_dtype,
                       void *stream);

/* ====================================================================================
 * AdamW over many tensors in one launch: beside sgd_step, for gradients as mlp_bwd
 * (fuse_sgd = 0) and expert_bwd store them.
 * ==================================================================================== */

/* One tensor of n >= 0 elements (all pointers to device memory, contiguous, aligned to their
 * elements). */
typedef struct {
    float *w;           /* fp32 master weights */
    uint16_t *w_lp;     /* bf16 copy of the updated weights, or NULL */
    const void *grad;   /* gradient, in grad_dtype */
    void *m, *v;        /* first and second moments: fp32, or one byte an element (state_bits 8) */
    float *m_scale;     /* state_bits 8: ceil(n/256) scales each, one for every 256 elements from */
    float *v_scale;     /* the tensor's first on; else unused */
    int64_t n;
    float decay;        /* weight decay, >= 0 */
    int grad_dtype;     /* IMBD_F32 or IMBD_BF16 */
    int state_bits;     /* 32 or 8 */
} imbd_adamw_tensor;

/* The plan of a set of tensors: adamw_plan writes it to HOST memory (plan_bytes from
 * adamw_plan_bytes; 0 for a bad argument or a set without elements), the caller copies it to
 * device memory (16-byte aligned) once and keeps both it and the tensors where they are. Tensors of
 * a set that share memory are refused (gradients, which are only read, may share theirs). */
size_t adamw_plan_bytes(const imbd_adamw_tensor *tensors, int n_tensors);
int adamw_plan(const imbd_adamw_tensor *tensors, int n_tensors, void *plan, size_t plan_bytes);

/* One step t on all tensors of a plan. With g = grad_scale * grad, in fp32 with every product and
 * sum rounded by itself:
 *   m <- beta1 m + (1 - beta1) g          v <- beta2 v + (1 - beta2) g^2
 *   w <- (1 - lr decay) w - lr/(1 - beta1^t) * m / (sqrt(v)/sqrt(1 - beta2^t) + eps)
 *   w_lp <- bf16(w)
 * (1 - beta, the bias corrections and 1 - lr*decay are formed in 64 bits.) t is `step` (>= 1), or
 * with step_dev != NULL the device int32 that it points to: a captured launch then follows the
 * caller's counter.
 * State of 8 bits, in blocks of 256 elements: m is held as float8 e4m3 times m_scale =
 * max|m| * (1/448) of the block, rounded to nearest, 448 at most; v as float8 e5m2 times v_scale =
 * max v * (1/57344), rounded up or down by a dither of the element's index and t (a second moment
 * that moves by 1 - beta2 a step would stay where it is if rounded to nearest), and never to zero:
 * what is positive and under the smallest normal number is held as that number (2^-14; where the
 * block's scale itself is 0 in fp32, m and v are 0). The update itself takes m and v before that
 * rounding. A NaN or an infinity in a gradient makes the element's state NaN or infinite, and with
 * 8-bit state its whole block's.
 * plan_bytes and n_tensors as at adamw_plan; plan_bytes == 0 is a no-op. 0 <= beta < 1, eps >= 0,
 * lr, eps and grad_scale finite, lr / (1 - beta1) finite and an eps above 0 not 0 in fp32 (with eps == 0
 * an element whose v is 0 becomes NaN or infinite, as the formula has it). A step_dev that holds less
 * than 1 is not noticed: 1 - beta^t is then 0 and the weights become NaN or infinite. */
int adamw_step(const void *plan, size_t plan_bytes, int n_tensors, double lr, double beta1,
               double beta2, double eps, float grad_scale, int step, const int32_t *step_dev,
               void *stream);

/* ====================================================================================
 * Options: kernel routing and K splits (for A/B timing and for tests that force a
 * route; the defaults are the measured choices)
 * ==================================================================================== */
enum imbd_option {
    IMBD_OPT_SKINNY_OFF = 0,    /* 1: forward / Delta_X products of B <= 256 on the tiled template */
    IMBD_OPT_SKINNY_SPLITS = 1, /* K split of the B <= 256 product kernel, 0 = planned (0..64) */
    IMBD_OPT_TOP_UNFUSED = 2,   /* 1: the top layer's softmax in a launch of its own */
    IMBD_OPT_WIDE_OFF = 3,      /* 1: forward / Delta_X products of B > 256 on the tiled template */
    IMBD_OPT_WIDE_SPLITS = 4,   /* K split of the B > 256 product kernel, 0 = planned */
    IMBD_OPT_DW_WIDE_MIN_K = 5, /* smallest batch whose fused update runs on the large-tile
                                   kernel (default 257) */
    IMBD_OPT_DW_STREAM = 6,     /* 0: past 256 samples the persistent update kernel reloads its
                                   Delta_Y block per 256 samples instead of streaming it */
    IMBD_OPT_DW_GENERIC = 7,    /* 1: the fused update on the tiled template */
    IMBD_OPT_GEMM_CFG = 8,      /* tile configuration of the tiled template, -1 = planned (-1..4) */
    IMBD_OPT_GEMM_SPLITS = 9,   /* K split of the tiled template, 0 = planned */
    IMBD_OPT_CONV_NT = 10,      /* 0: the conv tile on the tiled template; 1: on the large-tile
                                   kernels, tile height planned (default); 2 / 3: with tiles of
                                   at most 128 / 112 output positions */
    IMBD_OPT_SKINNY_NB = 11,    /* samples per workgroup of the B <= 256 product kernel, in units
                                   of 64 (1, 2 or 4), 0 = planned */
    IMBD_OPT_DW_WIDE_DUAL = 12, /* the large-tile fused update with two workgroups per CU
                                   (128-row tiles): 1 always, 0 never, -1 = planned (-1..1) */
    IMBD_OPT_LOCAL_PAIR = 13,   /* 0: the local backward pass's Delta_X and Delta_W products in two
                                   launches instead of one (default 1) */
    IMBD_OPT_REDUCE_TAIL = 14,  /* 0: a layer's Delta_X split-K reduce in a launch of its own instead
                                   of carried by that layer's update launch (default 1) */
    IMBD_OPT_COUNT = 15
};
/* Each option starts at the value of the environment variable named by
 * imbd_option_name(key) when the library is loaded (its default if unset or out of
 * range); the environment is not read again. imbd_set_option changes it for the whole
 * process: calls made afterwards use the new value. Options that move work between
 * kernels or change a K split change the workspace the *_workspace_bytes functions
 * report, so set them before sizing a workspace, and do not change them while another
 * thread has a call in flight. Returns IMBD_EINVAL for an unknown key or a value outside
 * the option's range. */
int imbd_set_option(int key, int value);
int imbd_get_option(int key, int *value);
/* The option's environment variable ("IMBD_..."), or "" for an unknown key. */
const char *imbd_option_name(int key);

/* ====================================================================================
 * Kernel timing (diagnostics for the roofline report)
 * ==================================================================================== */
enum imbd_kernel_class {
    IMBD_K_GEMM_FWD = 0, IMBD_K_GEMM_DX = 1, IMBD_K_GEMM_DW = 2, IMBD_K_SPLITK = 3,
    IMBD_K_SOFTMAX = 4, IMBD_K_BIAS = 5, IMBD_K_SGD = 6, IMBD_K_CAST = 7,
    IMBD_K_CONV_FWD = 8, IMBD_K_CONV_DGRAD = 9, IMBD_K_CONV_WGRAD = 10,
    IMBD_K_EXPERT_FWD = 11, IMBD_K_EXPERT_DX = 12, IMBD_K_EXPERT_DW = 13,
    IMBD_K_ROUTE = 14, IMBD_K_COMBINE = 15, IMBD_K_ADAMW = 16, IMBD_K_DISTILL = 17,
    IMBD_K_LOGPROBS = 18, IMBD_K_LINEAR = 19,
    IMBD_K_COUNT = 20
};
/* Start recording HIP events around every launch of kernel class `cls` whose layer tag
 * equals `layer` (-1: any layer), up to max_launches launches. Creates the events
 * (outside any compute call). The fused weight-gradient + update kernel takes the
 * events in its own dispatch (hipExtLaunchKernelGGL), so they hold its start and end
 * times; other launches get events enqueued before and after them. Returns IMBD_EINVAL
 * if a recording is already open. */
int imbd_timing_begin(int cls, int layer, int max_launches);
/* Stop recording, wait for the recorded events, and return the number of launches and
 * the summed kernel time in milliseconds. Destroys the events. */
int imbd_timing_end(int *n_launches, double *total_ms);

#ifdef __cplusplus
}
#endif
#endif /* IMBD_H */
