/*
 * bsa.h - C ABI of the Ball Sparse Attention (BSA) layer library for AMD MI355X (gfx950).
 *
 * The layer (arXiv 2506.12541, Section 2.2) orders an irregular point set with a ball
 * tree, then sums three attention branches over the ordered tokens, each scaled by a
 * sigmoid gate (Eq. 9): attention inside each ball (Ball Tree Attention, Eq. 3),
 * attention to MLP-compressed key/value blocks (Eq. 5), and attention to the top-k key
 * blocks selected per query group from the compressed scores (Eq. 6-8, 10-12).
 *
 * General conventions
 *  - Every pointer argument is a device pointer on the current HIP device unless stated
 *    otherwise. Every call is asynchronous on `stream` (a hipStream_t passed as void*;
 *    NULL = the default stream) and returns once its kernels are queued.
 *  - bsa_forward and bsa_backward run independent branches concurrently: on first use on
 *    a device the library creates one auxiliary stream (default priority) and two events
 *    for that device and keeps them until the process ends. (The forward of a bf16 layer
 *    without padding, whose ball and compressed attention share one launch, runs on
 *    `stream` alone.) Work on the auxiliary stream
 *    starts after an event recorded on `stream` and is joined back into `stream` before
 *    the call returns, so `stream` alone orders the call against the caller's other work.
 *    Calls from several threads are serialised while they enqueue. bsa_set_streams(1)
 *    runs every branch on `stream` instead (0: also without shared launches).
 *  - The library never allocates device memory and keeps no pointer after a call
 *    returns. The caller owns every buffer; sizes come from bsa_sizes() and
 *    bsa_ball_tree_workspace_bytes().
 *  - Arguments are validated on the host before anything is launched; an invalid call
 *    returns a non-zero status and launches nothing. A failed launch returns
 *    BSA_ERR_HIP. A fault inside a kernel surfaces at the caller's next synchronisation.
 *    bsa_last_error() gives a human-readable detail of the last failure on the calling
 *    thread. No C++ exception crosses this boundary.
 *  - Token layout: Q, K, V, O and their gradients are [B, H, N, d] row-major in ball
 *    order (slot order of the tree), so a ball, a compression block, a selection block
 *    and a query group of one head are each one contiguous run of rows.
 */
#ifndef BSA_H
#define BSA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  BSA_OK = 0,
  BSA_ERR_INVALID_ARGUMENT = 1,   /* a size, pointer or parameter is invalid            */
  BSA_ERR_UNSUPPORTED = 2,        /* valid but not implemented (e.g. head_dim not 32/64) */
  BSA_ERR_WORKSPACE_TOO_SMALL = 3,
  BSA_ERR_HIP = 4                 /* a HIP runtime call or kernel launch failed          */
} bsa_status_t;

typedef enum { BSA_F32 = 0, BSA_BF16 = 1 } bsa_dtype_t;
typedef enum { BSA_POOL_MLP = 0, BSA_POOL_MEAN = 1 } bsa_pool_t;
/* Coarse queries of the selection scores: the group mean of Eq. 11, or an MLP phi_q of
 * each block of l queries (Eq. 13). */
typedef enum { BSA_QC_MEAN = 0, BSA_QC_MLP = 1 } bsa_qcoarsen_t;

/* Layer hyper-parameters (notation of Section 2). */
typedef struct {
  int32_t batch;          /* B: independent point clouds                               */
  int32_t n;              /* N: token slots per cloud (power of two, >= 64)            */
  int32_t heads;          /* H                                                         */
  int32_t head_dim;       /* d: 32 or 64                                               */
  int32_t ball_size;      /* m: ball size of Eq. 3 (power of two, divides N)           */
  int32_t cmp_block;      /* l: compression block length of Eq. 5 (power of two)       */
  int32_t cmp_stride;     /* compression stride; must equal cmp_block (Eq. 5)          */
  int32_t slc_block;      /* l': selection block length of Eq. 8 (l'=r*l, r in 1,2,4;
                             multiple of 16; divides m)                                */
  int32_t topk;           /* k*: selected blocks per group (Eq. 7), 1..16; also
                             (16/g or 1) * k* * l' <= 4096                             */
  int32_t group_size;     /* g: query group size of Eq. 10: 1 (per-token selection, bf16
                             only) or a power of two >= 8 dividing m                   */
  int32_t mask_own_ball;  /* 1: a group may not select blocks of its own ball          */
  int32_t store_lse;      /* 1: the forward keeps each branch's log-sum-exp rows for the
                             backward; 0: they are not kept (saved.lse is NULL) and the
                             backward recomputes them by the branches' forward kernels
                             without the value products (same tiles and order: equal
                             to the stored rows bit for bit)                          */
  int32_t deterministic;  /* 0 or 1, no effect: every kernel is deterministic (no float
                             atomics; fixed-order sums), so both values give
                             bit-identical results                                     */
  int32_t kv_pool;        /* bsa_pool_t: MLP (default) or mean pooling of Eq. 5        */
  int32_t dtype;          /* bsa_dtype_t of Q, K, V, O, dO and the saved branch outputs */
  float softmax_scale;    /* 0 -> 1/sqrt(d)                                            */
  int32_t q_coarsen;      /* bsa_qcoarsen_t: BSA_QC_MEAN (default) or BSA_QC_MLP (Eq. 13-14;
                             needs group_size == cmp_block)                            */
  int32_t group_compression; /* 1: the compression branch attends from the coarse queries
                             and copies each result to the real queries of its block
                             (Eq. 15; needs group_size == cmp_block and n/cmp_block >= 64) */
} bsa_params_t;

/* One compression MLP phi (Eq. 5; also phi_q of Eq. 13): y = GELU_erf(x W1 + b1) W2 + b2
 * for the token-major flatten x of an l x d block (dummy rows zero). Float32, shared
 * across heads:
 * w1 [l*d, d], b1 [d], w2 [d, d], b2 [d], row-major. For bf16 layers w1 should hold
 * bf16-representable values: the first layer runs on bf16 matrix cores. */
typedef struct { const float *w1, *b1, *w2, *b2; } bsa_mlp_t;
typedef struct { float *w1, *b1, *w2, *b2; } bsa_mlp_grad_t;

/* Tensors the forward pass saves for the backward pass (all device, caller-owned).
 * bsa_saved_view() carves them out of one buffer of bsa_sizes()'s saved_bytes. */
typedef struct {
  int32_t* sel_idx;  /* [B, H, N/g, k*] selected block ids, ascending, -1 = empty slot  */
  float* lse;        /* [3, B, H, N] natural-log log-sum-exp per branch, -inf = no key;
                        NULL with store_lse = 0 (if set anyway, the forward fills it and
                        the backward still recomputes the rows)                         */
  void* o_branch;    /* [2, B, H, N, d] dtype: ball (0) and selection (1) outputs       */
  float* kcmp;       /* [B, H, N/l, d] compressed keys                                  */
  float* vcmp;       /* [B, H, N/l, d] compressed values                                */
  float* hid_k;      /* [B, H, N/l, d] hidden pre-activation of phi_k                   */
  float* hid_v;      /* [B, H, N/l, d] hidden pre-activation of phi_v                   */
  uint8_t* cvalid;   /* [B, N/l] 1 if the compression block holds a real token          */
  float* qcmp;       /* [B, H, N/g, d] coarse queries of the selection (Eq. 11 or 13)   */
  float* hid_q;      /* [B, H, N/l, d] hidden pre-activation of phi_q (BSA_QC_MLP)      */
  float* ocmp;       /* [B, H, N/l, d] coarse attention outputs of group compression    */
  float* o_cmp;      /* [B, H, N, d] float32 output of the compression branch. Kept
                        unrounded: the backward's softmax delta rowsum(dO o) comes from
                        it, and an error in that delta is common to every compressed key
                        of the query, so it would add up over the blocks in the
                        compression MLP's weight gradients                              */
} bsa_saved_t;

/* ---- Ball tree (Section 2.1 "Ball Tree Attention"; the ordering every branch uses) ---- */

/* Workspace bytes for bsa_build_ball_tree with these sizes (0 on invalid sizes). */
size_t bsa_ball_tree_workspace_bytes(int64_t n_real, int64_t n_pad, int32_t dim, int32_t batch);

/* Order each cloud by recursive median splits: a node of capacity C (a power of two)
 * holding the point set S splits on the axis of largest spread (max - min, formed in
 * float64; equal spreads -> lowest axis), its points ordered by (coordinate, index)
 * with -0.0 equal to +0.0; the first ceil(|S|/2) go to the left child (slots
 * [0, C/2)), the rest to the right child; recursion down to single slots.
 *   points: [batch, n_real, dim] float32, finite; dim = 3 (2 and 1 also accepted).
 *   perm:   [batch, n_pad] int32 output; slot -> point index within its cloud, -1 for a
 *           padding slot. 1 <= n_real <= n_pad, n_pad a power of two, n_pad <= 2^24.
 *   ws:     workspace of at least bsa_ball_tree_workspace_bytes() bytes. */
bsa_status_t bsa_build_ball_tree(const float* points, int64_t n_real, int32_t dim,
                                 int64_t n_pad, int32_t batch, int32_t* perm,
                                 void* ws, size_t ws_bytes, void* stream);

/* bsa_build_ball_tree without a workspace argument and without any device allocation, for
 * callers that cannot allocate (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc). Same arguments, ordering and errors as
 * bsa_build_ball_tree, minus ws / ws_bytes. The workspace is a static device array of the
 * library (10.7 MB on each device the library runs on, held until the process
 * ends) that covers batch * n_pad <= 131072 slots; larger sizes return
 * BSA_ERR_UNSUPPORTED and launch nothing. Every call on one device shares that array and
 * overwrites it: calls that overlap in time on one device (e.g. on two streams without
 * ordering between them) race and give wrong orderings; calls ordered on one stream are
 * safe. Nothing in the array needs clearing between calls (every word is written before
 * it is read). */
bsa_status_t bsa_build_ball_tree_noalloc(const float* points, int64_t n_real, int32_t dim, int64_t n_pad,
                                         int32_t batch, int32_t* perm, void* stream);

/* Gather per-point rows into ball order (the ordering step before Eq. 3):
 *   src  [batch, n_real, heads*head_dim] (dtype) -> dst [batch, heads, n_pad, head_dim],
 *   dst row = 0 where perm is -1. valid_out [batch, n_pad] (may be NULL) receives
 *   1 for real slots and 0 for padding. head_dim may be any value >= 1 (e.g. heads=1,
 *   head_dim=3 orders the gate logits). */
bsa_status_t bsa_permute(const void* src, const int32_t* perm, int64_t n_real, int64_t n_pad,
                         int32_t batch, int32_t heads, int32_t head_dim, int32_t dtype,
                         void* dst, uint8_t* valid_out, void* stream);

/* Inverse of bsa_permute: src [batch, heads, n_pad, head_dim] -> dst [batch, n_real,
 * heads*head_dim]; padding slots are dropped. dtype BSA_F32 or BSA_BF16. */
bsa_status_t bsa_unpermute(const void* src, const int32_t* perm, int64_t n_real, int64_t n_pad,
                           int32_t batch, int32_t heads, int32_t head_dim, int32_t dtype,
                           void* dst, void* stream);

/* ---- The layer (Section 2.2, Eq. 3, 5-12, 9) ---- */

/* Validate p and report the sizes of the forward workspace, the backward workspace and
 * the saved-tensor buffer. Any pointer may be NULL. */
bsa_status_t bsa_sizes(const bsa_params_t* p, size_t* ws_fwd_bytes, size_t* ws_bwd_bytes,
                       size_t* saved_bytes);

/* Point the fields of *out into the caller's buffer `base` of saved_bytes bytes
 * (256-byte aligned sub-buffers). Host-only arithmetic; launches nothing. */
bsa_status_t bsa_saved_view(const bsa_params_t* p, void* base, bsa_saved_t* out);

/* Forward pass.
 *   q, k, v: [B, H, N, d] dtype in ball order. valid: [B, N] uint8 (1 = real token) or
 *   NULL (all real). gate: [B, N, 3] float32 logits gamma_b in branch order (ball,
 *   compression, selection), shared across heads (Eq. 9). phi_k / phi_v: compression
 *   MLPs for keys / values (ignored for BSA_POOL_MEAN). phi_q: the query-coarsening MLP
 *   (read only for BSA_QC_MLP; may be NULL otherwise).
 *   o: [B, H, N, d] dtype output = sum_b sigmoid(gamma_b) * o_b; rows of padding slots 0.
 *   saved: filled for bsa_backward (and readable as per-branch outputs, LSE and the
 *   selected block ids). ws: at least ws_fwd_bytes. */
bsa_status_t bsa_forward(const bsa_params_t* p, const void* q, const void* k, const void* v,
                         const uint8_t* valid, const float* gate, const bsa_mlp_t* phi_k,
                         const bsa_mlp_t* phi_v, const bsa_mlp_t* phi_q, void* o,
                         const bsa_saved_t* saved, void* ws, size_t ws_bytes, void* stream);

/* Backward pass of bsa_forward given dO = d(loss)/d(o) ([B, H, N, d] dtype).
 * Outputs (overwritten, float32): dq, dk, dv [B, H, N, d]; dgate [B, N, 3];
 * dphi_k / dphi_v weight gradients summed over batch, heads and blocks (may be NULL for
 * BSA_POOL_MEAN). dphi_q: gradient of phi_q, which receives one only through group
 * compression (required for BSA_QC_MLP with group_compression = 1, else may be NULL and
 * is not written). No gradient flows through the top-k selection. Rows of padding slots
 * get zero gradients. ws: at least ws_bwd_bytes. */
bsa_status_t bsa_backward(const bsa_params_t* p, const void* q, const void* k, const void* v,
                          const uint8_t* valid, const float* gate, const bsa_mlp_t* phi_k,
                          const bsa_mlp_t* phi_v, const bsa_mlp_t* phi_q, const bsa_saved_t* saved,
                          const void* d_o, float* dq, float* dk, float* dv, float* dgate,
                          const bsa_mlp_grad_t* dphi_k, const bsa_mlp_grad_t* dphi_v,
                          const bsa_mlp_grad_t* dphi_q, void* ws, size_t ws_bytes, void* stream);

/* Streams used by bsa_forward and bsa_backward: 2 (default) = the caller's stream plus
 * the auxiliary stream (in the forward only where ball and compressed attention run as
 * separate launches), 1 = the caller's stream only (branches run one after another,
 * e.g. to time each alone), 0 = as 1, and the branches that otherwise share a launch
 * (ball and compressed attention forward, and their key-major backward passes, for bf16
 * layers without padding) get launches of their own, so that each branch can be timed.
 * Results are the same bit for bit in every mode. Process-wide; BSA_ERR_INVALID_ARGUMENT
 * for other values. */
bsa_status_t bsa_set_streams(int32_t n);

/* ---- The transformer block around the layer (Section 3.1) ----
 *
 * The paper's model stacks 18 blocks of RMSNorm, a BSA layer and a SwiGLU. One block, with
 * C = heads * head_dim channels and F SwiGLU hidden units, on tokens x [B, N, C] float32 in
 * ball order (padding rows zero):
 *   h = x + merge(BSA(Q, K, V; gate)) W_o^T,   [Q | K | V] = RMSNorm_1(x) W_qkv^T,
 *   gate = RMSNorm_1(x) W_g^T,   y = h + (silu(z W_1^T) * (z W_3^T)) W_2^T, z = RMSNorm_2(h),
 * RMSNorm(t) = t / sqrt(mean(t^2) + 1e-6) * gain; maps are bias-free and stored [out, in]
 * (head h of Q takes output columns h d .. h d + d - 1 of W_qkv, then K, then V).
 * Precision: bf16 layers only. The channel products take bf16 operands (round to nearest
 * even) and accumulate in float32; Q, K, V, the layer output, u = z W_1^T, w = z W_3^T
 * and silu(u) w are stored in bf16; the residual stream, the norms and the gate logits
 * (from the unrounded norm output and float32 W_g) are float32. In the backward pass the
 * gradients entering a product (dy, du, dw, dh, dO, dQ/dK/dV) are rounded to bf16.
 * Requirements beyond bsa_sizes: dtype BSA_BF16, C in {128, 256, 512, 1024}, F a positive
 * multiple of 128 (BSA_ERR_UNSUPPORTED otherwise). */
typedef struct {
  const float *g1;      /* [C]     gain of RMSNorm_1                                    */
  const float *wqkv;    /* [3C, C]                                                      */
  const float *wg;      /* [3, C]  gate logits (ball, compression, selection)           */
  const float *wo;      /* [C, C]                                                       */
  const float *g2;      /* [C]     gain of RMSNorm_2                                    */
  const float *w1, *w3; /* [F, C]                                                       */
  const float *w2;      /* [C, F]                                                       */
  bsa_mlp_t phi_k, phi_v, phi_q;  /* the layer's MLPs (phi_q read only for BSA_QC_MLP)  */
} bsa_block_weights_t;

/* Gradients of the weights (float32, same shapes, overwritten). phi_q: written only for
 * BSA_QC_MLP with group compression (as in bsa_backward). */
typedef struct {
  float *g1, *wqkv, *wg, *wo, *g2, *w1, *w3, *w2;
  bsa_mlp_grad_t phi_k, phi_v, phi_q;
} bsa_block_grads_t;

/* Tensors the block's forward pass saves for its backward pass (device, caller-owned;
 * bsa_block_saved_view() carves them out of one buffer). M = B * N token rows. */
typedef struct {
  bsa_saved_t layer;    /* the layer's own saved tensors                               */
  float* rstd1;         /* [M]        1 / rms of each row of x                          */
  float* rstd2;         /* [M]        1 / rms of each row of h                          */
  void* xn1;            /* [M, C]     bf16 RMSNorm_1(x)                                 */
  float* gate;          /* [B, N, 3]  gate logits                                       */
  void* q;              /* [B, H, N, d] bf16 (k, v likewise)                            */
  void* k;
  void* v;
  void* o;              /* [B, H, N, d] bf16 layer output                               */
  float* h;             /* [M, C]     residual stream after the attention sublayer      */
  void* xn2;            /* [M, C]     bf16 RMSNorm_2(h)                                 */
  void* uw;             /* [M, 2F]    bf16 u (columns 0..F-1) and w (F..2F-1)           */
  void* a;              /* [M, F]     bf16 silu(u) w                                    */
} bsa_block_saved_t;

/* Validate and report the forward workspace, backward workspace and saved-buffer sizes of
 * one block with F = ffn_dim. Any size pointer may be NULL. */
bsa_status_t bsa_block_sizes(const bsa_params_t* p, int32_t ffn_dim, size_t* ws_fwd_bytes,
                             size_t* ws_bwd_bytes, size_t* saved_bytes);

/* Point the fields of *out into `base` (saved_bytes of bsa_block_sizes). Host-only. */
bsa_status_t bsa_block_saved_view(const bsa_params_t* p, int32_t ffn_dim, void* base,
                                  bsa_block_saved_t* out);

/* Block forward: x [B, N, C] float32 -> y [B, N, C] float32 (y may not alias x). valid as
 * in bsa_forward. ws: at least ws_fwd_bytes. Asynchronous on `stream` (the layer inside
 * may also use the library's auxiliary stream, joined before return). */
bsa_status_t bsa_block_forward(const bsa_params_t* p, int32_t ffn_dim, const bsa_block_weights_t* w,
                               const float* x, const uint8_t* valid, float* y,
                               const bsa_block_saved_t* saved, void* ws, size_t ws_bytes, void* stream);

/* Block backward given dy = d(loss)/d(y) [B, N, C] float32: dx [B, N, C] float32 and the
 * weight gradients (summed over tokens in a fixed order; no float atomics). x and saved as
 * given to / filled by bsa_block_forward. ws: at least ws_bwd_bytes. */
bsa_status_t bsa_block_backward(const bsa_params_t* p, int32_t ffn_dim, const bsa_block_weights_t* w,
                                const float* x, const uint8_t* valid, const bsa_block_saved_t* saved,
                                const float* dy, float* dx, const bsa_block_grads_t* dw, void* ws,
                                size_t ws_bytes, void* stream);

/* ---- Dense operators beside the layer ----
 *
 * What a model has around the sparse layer: layer norms, affine maps with an activation or a
 * residual, gated maps, rotary positions with head norms, full attention over packed sequences, and
 * a cache of 8 bits for it. They follow the conventions above
 * (device pointers of the current device, asynchronous on `stream` alone, caller-owned
 * buffers, host-side checks before any launch) and are deterministic. They take bf16 or
 * float32 tensors (dtype); every sum and statistic is float32 and a result is rounded once to
 * its tensor's type. What is rounded to dtype on the way, into a matrix product or a tensor that is
 * kept, is named at each operator. Rows are contiguous along their last dimension; a leading
 * dimension or stride of 0 means the packed one. Outputs may not overlap inputs, except where
 * said. A call without rows (rows, m, total_q = 0) is valid; its weight gradients are zero. */

/* Layer norm over the last dimension: y = (x - mean) rstd gain + bias, rstd = 1 / sqrt(var + eps)
 * with the biased variance. */
typedef struct {
  int64_t rows;                       /* >= 0                                           */
  int32_t cols;                       /* 1 .. 32768                                     */
  int32_t dtype;                      /* bsa_dtype_t of x, y, dy and dx                 */
  float eps;                          /* > 0                                            */
  int64_t ld_x, ld_y, ld_dy, ld_dx;   /* elements between rows (0: cols)                */
} bsa_layernorm_t;

/* Validate p and report the backward workspace (ws_bwd_bytes may be NULL). */
bsa_status_t bsa_layernorm_sizes(const bsa_layernorm_t* p, size_t* ws_bwd_bytes);

/* x [rows, cols] -> y; gain, bias [cols] float32 (bias may be NULL: 0); mean, rstd [rows] float32
 * outputs, which the backward reads. */
bsa_status_t bsa_layernorm_forward(const bsa_layernorm_t* p, const void* x, const float* gain, const float* bias,
                                   void* y, float* mean, float* rstd, void* stream);

/* dx [rows, cols] (dtype), dgain and dbias [cols] float32 (dbias may be NULL: not formed), all
 * overwritten. dx may be dy or x (same leading dimension). */
bsa_status_t bsa_layernorm_backward(const bsa_layernorm_t* p, const void* x, const float* gain, const float* mean,
                                    const float* rstd, const void* dy, void* dx, float* dgain, float* dbias, void* ws,
                                    size_t ws_bytes, void* stream);

/* Affine map with an epilogue: z = x w^T + bias, y = act(z) + res, with x [m, k], w [n, k], y [m, n].
 * float32 products (all but those of a forward of few rows) are formed from three bf16 parts of each
 * value: it enters them within 2^-24 of itself or, where it is smaller than 2^-110, within 2^-134.
 * GELU of bf16 tensors evaluates erfc to 1.5e-7 absolute: 5e-4 of the result at z = -4, 4e-3 (a
 * bf16 rounding) at z = -6. */
typedef enum { BSA_ACT_NONE = 0, BSA_ACT_RELU = 1, BSA_ACT_GELU = 2 /* erf form */, BSA_ACT_SILU = 3 } bsa_act_t;
typedef struct {
  int64_t m;                            /* rows, 0 .. 2^31 - 256                        */
  int32_t k, n;                         /* input and output channels, 1 .. 2^24; x, y
                                           and w have fewer than 2^24 tiles of 128 x 128 */
  int32_t dtype;                        /* bsa_dtype_t of every tensor                  */
  int32_t act;                          /* bsa_act_t                                    */
  int64_t ld_x, ld_w, ld_y, ld_res, ld_dy;  /* elements between rows (0: packed)        */
} bsa_linear_t;

/* Validate p and report the workspaces (pointers may be NULL). */
bsa_status_t bsa_linear_sizes(const bsa_linear_t* p, size_t* ws_fwd_bytes, size_t* ws_bwd_bytes);

/* bias [n], res [m, n] (may be y itself) and pre may be NULL. pre [m, n] packed receives z for the
 * backward of a map with an activation (z rounded to dtype). */
bsa_status_t bsa_linear_forward(const bsa_linear_t* p, const void* x, const void* w, const void* bias, const void* res,
                                void* y, void* pre, void* ws, size_t ws_bytes, void* stream);

/* With dz = dy act'(z): dx = dz w [m, k], dw = dz^T x [n, k], db = sum of dz over the rows [n], all
 * dtype, packed and overwritten; each may be NULL (not formed). The residual's gradient is dy.
 * pre: as filled by the forward (ignored, may be NULL, without an activation). dz is rounded to
 * dtype where it enters the products (not in db). */
bsa_status_t bsa_linear_backward(const bsa_linear_t* p, const void* x, const void* w, const void* pre, const void* dy,
                                 void* dx, void* dw, void* db, void* ws, size_t ws_bytes, void* stream);

/* Gated map: [g | u] = x w^T + bias, y = act(g) u, with x [m, k], w [2 n, k] (the n rows of the gate's map, then
 * those of the other), bias [2 n], y [m, n]. Products as the affine map's. */
typedef struct {
  int64_t m;                            /* rows, 0 .. 2^31 - 256                        */
  int32_t k, n;                         /* input and output channels, 1 .. 2^24 and 2^23; x, y
                                           and w have fewer than 2^24 tiles of 128 x 128 */
  int32_t dtype;                        /* bsa_dtype_t of every tensor                  */
  int32_t act;                          /* bsa_act_t                                    */
  int64_t ld_x, ld_w, ld_y, ld_dy;      /* elements between rows (0: packed)            */
} bsa_gated_t;

/* Validate p and report the workspaces (pointers may be NULL), which begin on 16 bytes. */
bsa_status_t bsa_gated_sizes(const bsa_gated_t* p, size_t* ws_fwd_bytes, size_t* ws_bwd_bytes);

/* bias and pre may be NULL. pre [m, 2 n] packed receives [g | u] for the backward, rounded to dtype. */
bsa_status_t bsa_gated_forward(const bsa_gated_t* p, const void* x, const void* w, const void* bias, void* y, void* pre,
                               void* ws, size_t ws_bytes, void* stream);

/* With dz = [dy u act'(g) | dy act(g)]: dx = dz w [m, k], dw = dz^T x [2 n, k], db = sum of dz over the rows
 * [2 n], all dtype, packed and overwritten; each may be NULL (not formed). pre: as filled by the forward.
 * dz is rounded to dtype where it enters the products (not in db). */
bsa_status_t bsa_gated_backward(const bsa_gated_t* p, const void* x, const void* w, const void* pre, const void* dy, void* dx,
                                void* dw, void* db, void* ws, size_t ws_bytes, void* stream);

/* Rotary positions of queries q [rows, heads, head_dim] and keys k [rows, kv_heads, head_dim], with the norm of
 * each head in the same pass. With a gain [head_dim] (float32) n = x / sqrt(mean(x^2) + eps) gain, without (NULL)
 * n = x. The first rot values of a head are rot / 2 pairs: (i, i + rot / 2), or with interleaved (2 i, 2 i + 1); pair
 * i turns by t = position * freq[i], y = magnitude (n_a cos t - n_b sin t, n_a sin t + n_b cos t). The rest of
 * n passes. positions [rows, axes]: axis a turns the pairs [a, a + 1) (rot / 2) / axes. Angles are formed and
 * reduced in 64 bits (meant for |t| < 2^31), cosines and sines are float32, off by 2^-23 at most. */
typedef enum { BSA_POS_I32 = 0, BSA_POS_F32 = 1 } bsa_pos_t;
typedef struct {
  int64_t rows;                         /* 0 .. 2^40                                    */
  int32_t heads, kv_heads;              /* >= 1; kv_heads 0: no keys (their pointers are not read) */
  int32_t head_dim;                     /* 2 .. 256                                     */
  int32_t rot;                          /* even, 2 .. head_dim                          */
  int32_t axes;                         /* 1 .. 4, divides rot / 2                      */
  int32_t pos_type;                     /* bsa_pos_t                                    */
  int32_t interleaved;                  /* 0 or 1                                       */
  int32_t dtype;                        /* bsa_dtype_t of q, k, y and their gradients   */
  float eps;                            /* > 0 (read with a gain)                       */
  float magnitude;                      /* finite, > 0                                  */
  /* elements between rows and between heads; both 0: packed. o: the outputs (y, or in the backward
   * the gradients of q and k); d: dy */
  int64_t q_row, q_head, k_row, k_head, oq_row, oq_head, ok_row, ok_head, dq_row, dq_head, dk_row, dk_head;
} bsa_rotary_t;

/* Validate p and report the backward workspace (ws_bwd_bytes may be NULL). */
bsa_status_t bsa_rotary_sizes(const bsa_rotary_t* p, size_t* ws_bwd_bytes);

/* freq [rot / 2] float64. y_q may be q and y_k may be k (same strides). */
bsa_status_t bsa_rotary_forward(const bsa_rotary_t* p, const void* q, const void* k, const void* positions, const double* freq,
                                const float* gain_q, const float* gain_k, void* y_q, void* y_k, void* stream);

/* dq and dk (dtype), dgain_q and dgain_k [head_dim] float32 (each may be NULL: not formed), given dy_q and dy_k. q is
 * read only with gain_q, k only with gain_k (else they may be NULL), as they were before the forward. dq may
 * be dy_q or q, dk may be dy_k or k (same strides). */
bsa_status_t bsa_rotary_backward(const bsa_rotary_t* p, const void* q, const void* k, const void* positions, const double* freq,
                                 const float* gain_q, const float* gain_k, const void* dy_q, const void* dy_k, void* dq,
                                 void* dk, float* dgain_q, float* dgain_k, void* ws, size_t ws_bytes, void* stream);

/* Full attention over packed sequences with grouped heads. Sequence s has the query rows
 * [cu_q[s], cu_q[s+1]) and the key rows [cu_k[s], cu_k[s] + l), l = used_k[s] (a cache that is
 * filled so far) or, with used_k NULL, cu_k[s+1] - cu_k[s]. Query head h reads key head
 * h / (heads / kv_heads). o = softmax(scale q k^T) v over the visible keys: all of the sequence's, or,
 * causal, key j for query i when j <= i + (l - query rows): the last query sees every key. A query
 * that sees no key has o = 0 and lse = -inf and takes no part in the gradients. Probabilities enter the
 * products with v, d_o and (in a correction of dq) k, and dS those with k and q, rounded to dtype; o
 * enters dq and dk as it was rounded, with that rounding taken out. A value that is not
 * finite reaches rows and keys that see it (where it may become NaN in all columns), and no others.
 * cu_q, cu_k [seqs + 1] and used_k [seqs] are device arrays (int32): from 0, not decreasing, at most
 * total_q, total_k and the capacity cu_k[s+1] - cu_k[s]. They cannot be checked on the host: values
 * outside the tensors are pulled inside (nothing is read or written out of bounds), and then
 * the outputs are not defined. */
typedef struct {
  int32_t seqs;                         /* 1 .. 2^22 (more: where the tiles of a launch,
                                           seqs and one for every 16 rows, are < 2^24)  */
  int32_t heads, kv_heads;              /* kv_heads divides heads                       */
  int32_t head_dim;                     /* 32, 64 or 128                                */
  int64_t total_q, total_k;             /* rows of q and of k and v; total_q times
                                           heads / kv_heads and total_k <= 2^30         */
  int32_t causal;                       /* 0 or 1                                       */
  int32_t dtype;                        /* bsa_dtype_t of q, k, v, o, d_o, dq, dk, dv   */
  float softmax_scale;                  /* 0 -> 1/sqrt(head_dim)                        */
  int32_t zero_rest;                    /* rows in no sequence (and unused cache rows):
                                           0 = outputs keep what they held, 1 = outputs
                                           are set to 0 (lse to -inf)                   */
  /* elements between rows and between heads of [rows, heads, head_dim] tensors; multiples of
   * 16 bytes, like the tensors' addresses; both 0: packed */
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, do_row, do_head;
} bsa_attention_t;

/* Validate p and report the workspaces (pointers may be NULL). */
bsa_status_t bsa_attention_sizes(const bsa_attention_t* p, size_t* ws_fwd_bytes, size_t* ws_bwd_bytes);

/* o [total_q, heads, head_dim], lse [heads, total_q] float32 (natural logarithm). */
bsa_status_t bsa_attention_forward(const bsa_attention_t* p, const void* q, const void* k, const void* v,
                                   const int32_t* cu_q, const int32_t* cu_k, const int32_t* used_k, void* o, float* lse,
                                   void* ws, size_t ws_bytes, void* stream);

/* dq [total_q, heads, head_dim], dk and dv [total_k, kv_heads, head_dim], packed, dtype, overwritten (a
 * key head's gradient is the sum over its group). o and lse as filled by the forward. Sequences may
 * not share rows. */
bsa_status_t bsa_attention_backward(const bsa_attention_t* p, const void* q, const void* k, const void* v,
                                    const void* o, const float* lse, const void* d_o, const int32_t* cu_q,
                                    const int32_t* cu_k, const int32_t* used_k, void* dq, void* dk, void* dv, void* ws,
                                    size_t ws_bytes, void* stream);

/* Cache of 8 bits. A cache holds keys, and values, as e4m3 bytes [total_k, kv_heads, head_dim] and an exponent
 * code for each row and key head [kv_heads, total_k]: a byte stands for its e4m3 value times 2^(code - 127). A row
 * of a head is written with the smallest exponent code - 127 in [-64, 63] at which its largest magnitude is at
 * most 448 times the scale (values past 448 2^63 are cut to it), each value rounded to nearest even, which is
 * the only rounding. Infinities and NaN are written as NaN and take no part in the scale.
 * Sequence s owns the cache rows [cu_k[s], cu_k[s+1]), of which the first l = used_k[s] are in use (NULL: all).
 * Its n = cu_q[s+1] - cu_q[s] rows of k and v [rows, kv_heads, head_dim] are the last n of those l; rows that would
 * lie before the sequence's first are not written, and are read as 0. The arrays of offsets are as
 * bsa_attention_forward takes them. */
typedef struct {
  int32_t seqs;                         /* 1 .. 2^24                                    */
  int32_t kv_heads;                     /* 1 .. 65535                                   */
  int32_t head_dim;                     /* 32, 64 or 128                                */
  int32_t dtype;                        /* bsa_dtype_t of k and v                       */
  int64_t rows, total_k;                /* rows of k and v, and of the cache; <= 2^30   */
  /* elements between rows and between heads of k and v, bytes between those of the cache's keys (ck) and
   * values (cv); multiples of 16 bytes, like the tensors' addresses; both 0: packed */
  int64_t k_row, k_head, v_row, v_head, ck_row, ck_head, cv_row, cv_head;
} bsa_cache_t;

/* New rows into the cache. exp_k and exp_v: the exponent codes. */
bsa_status_t bsa_cache_write(const bsa_cache_t* p, const void* k, const void* v, const int32_t* cu_q, const int32_t* cu_k,
                             const int32_t* used_k, void* cache_k, void* cache_v, uint8_t* exp_k, uint8_t* exp_v, void* stream);

/* Rows back from the cache: the values their bytes stand for, exactly; rows in no sequence are 0. */
bsa_status_t bsa_cache_read(const bsa_cache_t* p, const void* cache_k, const void* cache_v, const uint8_t* exp_k,
                            const uint8_t* exp_v, const int32_t* cu_q, const int32_t* cu_k, const int32_t* used_k, void* k,
                            void* v, void* stream);

/* bsa_attention_forward with the cache for k and v: o = softmax(scale q K^T) V with the values that the bytes stand
 * for. Everything else is as there, p's k and v strides being those of the cache in bytes; there is no backward.
 * bf16 queries: probabilities enter the product with V as two bf16 parts (within 2^-16 of themselves) in calls of few
 * rows, such as single tokens, and rounded to bf16 in others. float32 queries, and their
 * probabilities, enter the products as three bf16 parts (within 2^-24 of themselves; a query value past the
 * largest bf16 number gives NaN). */
bsa_status_t bsa_cache_attention_sizes(const bsa_attention_t* p, size_t* ws_bytes);
bsa_status_t bsa_cache_attention_forward(const bsa_attention_t* p, const void* q, const void* cache_k, const void* cache_v,
                                         const uint8_t* exp_k, const uint8_t* exp_v, const int32_t* cu_q, const int32_t* cu_k,
                                         const int32_t* used_k, void* o, float* lse, void* ws, size_t ws_bytes, void* stream);

/* ---- Measurement support (not part of the layer's computation) ---- */

/* on = 1: start recording, clearing earlier records; on = 0: stop and clear. While on,
 * every timed phase of the library records a start and a stop HIP event on the stream
 * its kernels are launched on (phases on the two streams of a call may overlap in time). Phases: "tree", "permute", "fwd.compress", "fwd.select",
 * "fwd.ball", "fwd.cmp", "fwd.slc", "fwd.gate", "bwd.lse" (store_lse = 0), "bwd.gate", "bwd.dq_ball", "bwd.dq_cmp",
 * "bwd.dq_slc", "bwd.kv_ball", "bwd.kv_cmp", "bwd.mlp", "bwd.slc_csr", "bwd.slc_kv", and
 * for the block "blk.norm", "blk.gemm" (activation products), "blk.wgrad" (weight
 * gradients), "blk.elem" (SwiGLU, casts, layout changes). Each dense operator's call is one
 * phase: "norm.fwd", "norm.bwd", "linear.fwd", "linear.bwd", "gated.fwd", "gated.bwd",
 * "rotary.fwd", "rotary.bwd", "attn.fwd", "attn.bwd", "cache.write", "cache.read", "cache.attn".
 * Host-side bookkeeping only; no device memory is allocated. */
bsa_status_t bsa_timing_enable(int32_t on);

/* Restrict the recording to the comma-separated phase names in `phases` (NULL or "" =
 * every phase), so that a measured region carries the events of the phases it reports
 * and no others. Host-side bookkeeping only. */
bsa_status_t bsa_timing_select(const char* phases);

/* Sum of the recorded durations of `phase` (milliseconds) and the number of records;
 * waits for the recorded events to complete. */
bsa_status_t bsa_timing_query(const char* phase, double* total_ms, int32_t* count);

const char* bsa_status_string(bsa_status_t s);
/* Detail of the last failure on the calling thread ("" if none). */
const char* bsa_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* BSA_H */
