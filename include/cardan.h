/*
 * cardan.h -- C ABI of libcardan.so, an MI355X (gfx950) implementation of one
 * batch-1-to-64 Mixture-of-Experts decode layer whose expert matrices are
 * stored compressed.
 *
 * The layer (paper Sec. 2.1): a router scores the E experts for every token,
 * keeps the top-k and weights them with a softmax over the k kept logits;
 * every kept expert runs gate and up projections, the SiLU-gated product
 * p = silu(g) * u, and a down projection; the layer output is the
 * affinity-weighted sum of the expert outputs.
 *
 * Expert representation (paper Sec. 2.3 and Sec. 3.1, Eq. (1)): a gate or up
 * matrix W_e [H, I] is Q_B(J_e) + U V_e, where Q_B(J_e) is rebuilt from a
 * shared code book B [K, d] and a private uint8 index map J_e [H/d, I] (block
 * b of column j is code word J_e[b, j], whose element i sits at input row
 * b*d + i), U [H, r] is a basis shared by all experts and V_e [r, I] holds
 * private coefficients. The down matrix [I, H] is Q_B(J^d_e) + A_e B with
 * private A_e [I, r] and a shared output-side basis B [r, H].
 *
 * Conventions for every entry point:
 *   - bf16 values are raw bit patterns (uint16_t); all arrays are dense and
 *     row-major in the shapes given; every pointer is a DEVICE pointer,
 *     16-byte aligned, owned by the caller and only read during the call
 *     (outputs are written). The library never allocates, frees or
 *     synchronises inside these calls and keeps no pointer after returning.
 *   - All work is enqueued on `stream` and the call returns without waiting.
 *     Buffers must stay valid until the stream has passed the work.
 *   - Arguments are validated before anything is enqueued; on any error
 *     nothing is launched, a negative code is returned and
 *     cardan_last_error() describes it.
 *   - `ws` is a caller-owned device workspace of at least
 *     cardan_workspace_bytes() bytes. It must be zero-filled once before its
 *     first use; every completed call leaves it ready for the next. Calls
 *     that overlap in time must not share a workspace.
 *   - Supported shapes: d in {2, 4, 8}; 1 <= K <= 256; H % 64 == 0;
 *     I % 32 == 0; 1 <= E <= 1024; 1 <= top_k <= min(E, 32); 0 <= r <= 512;
 *     1 <= B <= 64. Other shapes return CARDAN_ERR_UNSUPPORTED or
 *     CARDAN_ERR_BAD_SHAPE.
 *   - Code values >= K read zero code words (memory-safe); expert indices
 *     outside [0, E) passed to cardan_vq_lr_expert_ffn contribute nothing.
 *   - The first int32 of the workspace (CARDAN_WS_STATUS_OFFSET) counts
 *     internal waits that gave up after their bound (seconds); nonzero means
 *     the results of the calls since it was last zero are invalid. The
 *     library never clears it; the caller may.
 *   - The layer kernels are persistent: each launches at most as many
 *     workgroups as the device holds at once and their work items wait on
 *     one another. They need the device's compute units to themselves while
 *     they run; other resident work (another stream or process) can keep
 *     workgroups from starting, and the waits that depend on them then give
 *     up into the status count above (the results are invalid, nothing hangs).
 *   - A workspace serves one (H, I, E): its counter offsets depend on those
 *     three only, so calls of any batch, rank, block length or expert-weight
 *     form on that shape may share it in turn; zero it again before using it
 *     for another (H, I, E).
 *   - Reentrancy: the entry points keep no mutable host state apart from the
 *     thread-local error text and an occupancy cache guarded by a mutex; host
 *     threads may call them concurrently on separate workspaces. The
 *     profiling hooks below are the exception (host-global, not thread-safe).
 */
#ifndef CARDAN_H
#define CARDAN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Same declaration as HIP's own; lets this header stand alone. */
typedef struct ihipStream_t* hipStream_t;
typedef struct ihipEvent_t* hipEvent_t;

#define CARDAN_ABI_VERSION 1
#define CARDAN_WS_STATUS_OFFSET 0

enum {
  CARDAN_OK = 0,
  CARDAN_ERR_NULL_PTR = -1,   /* a required pointer is NULL               */
  CARDAN_ERR_BAD_SHAPE = -2,  /* shape or batch outside the valid domain  */
  CARDAN_ERR_UNSUPPORTED = -3,/* valid but not compiled (e.g. d == 16)    */
  CARDAN_ERR_WORKSPACE = -4,  /* ws_bytes below cardan_workspace_bytes()  */
  CARDAN_ERR_HIP = -5,        /* a HIP launch or event call failed        */
  CARDAN_ERR_ALIGN = -6       /* a pointer is not 16-byte aligned         */
};

typedef uint16_t cardan_bf16;

/* Layer shape: hidden size H, expert intermediate size I, E experts, top_k
 * selected per token, VQ block length d, K code words, rank r (Table 1). */
typedef struct {
  int32_t H, I, E, top_k, d, K, r;
} cardan_shape;

/* One layer's weights (device pointers). With r == 0 the six low-rank
 * pointers may be NULL. U_up may equal U_gate (one basis for both). */
typedef struct {
  const cardan_bf16* router_w;    /* [H][E]                                  */
  const float*       router_bias; /* [E] added to the logits, or NULL        */
  const cardan_bf16* cb_gate;     /* [K][d] shared gate code book            */
  const cardan_bf16* cb_up;       /* [K][d] shared up code book              */
  const cardan_bf16* cb_down;     /* [K][d] shared down code book            */
  const uint8_t*     codes_gate;  /* [E][H/d][I] private index maps          */
  const uint8_t*     codes_up;    /* [E][H/d][I]                             */
  const uint8_t*     codes_down;  /* [E][I/d][H]                             */
  const cardan_bf16* U_gate;      /* [H][r] shared basis (gate)              */
  const cardan_bf16* U_up;        /* [H][r] shared basis (up)                */
  const cardan_bf16* V_gate;      /* [E][r][I] private coefficients          */
  const cardan_bf16* V_up;        /* [E][r][I]                               */
  const cardan_bf16* A_down;      /* [E][I][r] private down factor           */
  const cardan_bf16* B_down;      /* [r][H] shared output-side down basis    */
} cardan_layer;

/* ABI version of the loaded library (CARDAN_ABI_VERSION). */
int cardan_abi_version(void);

/* Text of the last error on the calling thread ("" if none). Valid until the
 * next cardan_* call on the same thread. */
const char* cardan_last_error(void);

/* Workspace size in bytes needed by every ws-taking entry point for this
 * shape and any batch up to B (the dense-weight entry points and the decode
 * step included).
 * Host-only; no device is touched. */
int cardan_workspace_bytes(const cardan_shape* shape, int32_t B, size_t* out);

/* Router and gating (paper Sec. 2.1): logits l[t][e] = sum_h x[t][h] *
 * router_w[h][e] + router_bias[e], accumulated in float64 from the exact bf16
 * products; the top_k experts by descending logit (exact ties to the lower
 * index) go to topk_idx[B][top_k] (int32, in that order) and their softmax
 * over the top_k logits to topk_w[B][top_k] (float32).
 * x: [B][H] bf16. */
int cardan_route_topk(const cardan_shape* shape, int32_t B, const cardan_bf16* x,
                      const cardan_bf16* router_w, const float* router_bias,
                      int32_t* topk_idx, float* topk_w,
                      void* ws, size_t ws_bytes, hipStream_t stream);

/* Shared projections of Eq. (1) (paper Sec. 4.2, computed once per token):
 * z[0][t][q] = sum_h U_gate[h][q] x[t][h] and z[1][t][q] likewise with U_up,
 * as float32 z[2][B][r]. Both halves are always written; U_up may equal
 * U_gate. Requires r > 0. */
int cardan_shared_proj(const cardan_shape* shape, int32_t B, const cardan_bf16* x,
                       const cardan_bf16* U_gate, const cardan_bf16* U_up, float* z,
                       void* ws, size_t ws_bytes, hipStream_t stream);

/* Expert computation and weighted combine for a given routing (Sec. 2.1,
 * Eq. (1)): tokens are grouped by expert so each selected expert's codes are
 * read once; for every (token, selected expert) g and u are the VQ gather sum
 * plus V^T z (one float32 accumulation), p = silu(g) * u, the down output is
 * Q^T p + B^T (A^T p), and y[t] = sum_j topk_w[t][j] * y_{topk_idx[t][j]}.
 * topk_idx/topk_w: [B][top_k] as produced by cardan_route_topk; z: [2][B][r]
 * as produced by cardan_shared_proj (may be NULL iff r == 0);
 * y: [B][H] float32 output. */
int cardan_vq_lr_expert_ffn(const cardan_shape* shape, int32_t B, const cardan_bf16* x,
                            const int32_t* topk_idx, const float* topk_w, const float* z,
                            const cardan_layer* layer, float* y,
                            void* ws, size_t ws_bytes, hipStream_t stream);

/* The whole layer (paper Sec. 2.1 with the experts of Sec. 3.1, Eq. (1), and
 * the once-per-token shared projections and cross-expert batching of
 * Sec. 4.2): route + top-k + gating as cardan_route_topk, z = U^T x as
 * cardan_shared_proj, then the grouped expert computation and weighted
 * combine of cardan_vq_lr_expert_ffn. Writes y [B][H] float32 and the
 * routing topk_idx [B][top_k] int32, topk_w [B][top_k] float32.
 * Gate/up form: the VQ part is decoded from code words on the matrix cores;
 * with the environment variable CARDAN_GATEUP=tbook (read at every call of
 * this entry point and of cardan_moe_layer_relu2) one-token experts sum the
 * per-token projection code book T[b][k] = x_b . cb_k of Sec. 4.2 instead
 * (d = 4 or 8, K a multiple of 4, at most 64 MiB of T; otherwise the code
 * words). Both give the same result up to float32 rounding. */
int cardan_moe_layer(const cardan_shape* shape, int32_t B, const cardan_bf16* x,
                     const cardan_layer* layer, float* y, int32_t* topk_idx, float* topk_w,
                     void* ws, size_t ws_bytes, hipStream_t stream);

/* The whole layer with up-only experts and a squared-ReLU activation (the
 * expert form of the paper's Nemotron-3 model, Table 2 "up" and the fidelity
 * test of Sec. 5.7): routing and z = U_up^T x as cardan_moe_layer, then for
 * every (token, selected expert) u = VQ gather sum + V_up^T z, p =
 * max(u, 0)^2, the down output Q^T p + B^T (A^T p), and the weighted combine.
 * The gate fields of `layer` (cb_gate, codes_gate, U_gate, V_gate) are not
 * read and may be NULL. Outputs, workspace and errors as cardan_moe_layer. */
int cardan_moe_layer_relu2(const cardan_shape* shape, int32_t B, const cardan_bf16* x,
                           const cardan_layer* layer, float* y, int32_t* topk_idx, float* topk_w,
                           void* ws, size_t ws_bytes, hipStream_t stream);

/* One decode step through n_layers stacked MoE layers (the 48-layer workload
 * of the paper's Qwen3 decoding, attention omitted): layer 0 reads x0
 * [B][H] bf16; layer l + 1 reads x_{l+1} = bf16_rne(y_l / sqrt(mean_h(y_l^2)
 * + eps)) of layer l's output y_l (no learned scale), as cardan_rmsnorm_bf16
 * would form it; y [B][H] float32 receives the last layer's output. Every
 * layer is cardan_moe_layer on its own weights layers[l] (Sec. 2.1, Sec. 3.1
 * Eq. (1), Sec. 4.2), all with the same shape. Per layer l the routing goes
 * to topk_idx / topk_w [n_layers][B][top_k]; x_norm, if not NULL, receives
 * the normalised inputs of layers 1..n_layers-1 as [n_layers - 1][B][H] bf16.
 * The normalisation runs inside the next layer's routing kernel (the layer's
 * combine writes per-token partial sums of y^2), so a layer costs two kernel
 * launches. With the environment variable CARDAN_PREFETCH set to "1" the
 * expert kernel's idle workgroups also read the next layer's router weights,
 * bases and code books ahead of its routing kernel (the paper's overlap of
 * routing-independent reads, Sec. 4.1); it changes no output and is off by
 * default because it measured slower. ws: at least
 * cardan_workspace_bytes(shape, B) bytes; one workspace serves every layer.
 * 1 <= n_layers <= 4096, eps finite and >= 0. */
int cardan_moe_decode_step(const cardan_shape* shape, int32_t B, int32_t n_layers, const cardan_bf16* x0,
                           const cardan_layer* layers, float eps, float* y, cardan_bf16* x_norm,
                           int32_t* topk_idx, float* topk_w, void* ws, size_t ws_bytes,
                           hipStream_t stream);

/* Size of the library's own scratch array, one per GPU (16 MiB). */
#define CARDAN_SCRATCH_BYTES (16u << 20)

/* cardan_moe_layer without a workspace argument, for callers that cannot
 * allocate device memory: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc. The kernels use a fixed device-resident
 * scratch array of CARDAN_SCRATCH_BYTES inside the library (each GPU the
 * library runs on holds its own copy until the process ends); this call
 * allocates nothing (no hipMalloc, hipFree or allocating library routine).
 * Arguments, outputs, results and errors are those of cardan_moe_layer; a
 * layer whose workspace at this batch exceeds the array returns
 * CARDAN_ERR_WORKSPACE before anything is enqueued.
 * Every call on a GPU shares that GPU's array, which keeps the last call's
 * contents: calls that overlap in time on one GPU (several streams or host
 * threads) race and give undefined results, so serialise them. A call whose
 * (H, I, E) differs from the previous call's on the GPU, the first call, and
 * any call recorded under graph capture enqueue a small zero-fill kernel of
 * the array's counters before the layer. The wait-timeout status count of
 * these calls is not readable (cardan_moe_layer with a workspace reports it). */
int cardan_moe_layer_noalloc(const cardan_shape* shape, int32_t B, const cardan_bf16* x,
                             const cardan_layer* layer, float* y, int32_t* topk_idx,
                             float* topk_w, hipStream_t stream);

/* Dense bf16 expert weights of an uncompressed layer (device pointers). */
typedef struct {
  const cardan_bf16* router_w;    /* [H][E]                                  */
  const float*       router_bias; /* [E] added to the logits, or NULL        */
  const cardan_bf16* W_gate;      /* [E][H][I]                               */
  const cardan_bf16* W_up;        /* [E][H][I]                               */
  const cardan_bf16* W_down;      /* [E][I][H]                               */
} cardan_dense_layer;

/* The layer with compressed gate and up projections (Eq. (1)) and a dense
 * bf16 down projection W_down [E][I][H], the form whose down matrices the
 * paper leaves uncompressed (Sec. 3.1): routing as cardan_route_topk, g and
 * u as in cardan_vq_lr_expert_ffn, then y[t] = sum_j topk_w[t][j] *
 * W_down[e_j]^T p_j. The layer's cb_down, codes_down, A_down and B_down are
 * not read (may be NULL). Outputs as cardan_moe_layer. H * I * 2 must stay
 * below 2^31 (CARDAN_ERR_UNSUPPORTED otherwise). */
int cardan_moe_layer_dense_down(const cardan_shape* shape, int32_t B, const cardan_bf16* x,
                                const cardan_layer* layer, const cardan_bf16* W_down, float* y,
                                int32_t* topk_idx, float* topk_w,
                                void* ws, size_t ws_bytes, hipStream_t stream);

/* The uncompressed MoE layer (paper Sec. 2.1), the baseline the compressed
 * form is measured against: routing as cardan_route_topk, then for every
 * (token, selected expert) p = silu(W_gate[e]^T x) * (W_up[e]^T x) and
 * y[t] = sum_j topk_w[t][j] * W_down[e_j]^T p_j, float32 accumulation.
 * Only H, I, E and top_k of `shape` are read; the workspace size is
 * cardan_workspace_bytes() of any valid shape with those four fields.
 * H * I * 2 must stay below 2^31. Outputs as cardan_moe_layer. */
int cardan_dense_moe_layer(const cardan_shape* shape, int32_t B, const cardan_bf16* x,
                           const cardan_dense_layer* layer, float* y, int32_t* topk_idx,
                           float* topk_w, void* ws, size_t ws_bytes, hipStream_t stream);

/* The uncompressed layer with up-only squared-ReLU experts (Table 2, "up"):
 * as cardan_dense_moe_layer with p = max(W_up[e]^T x, 0)^2; W_gate is not
 * read (may be NULL). */
int cardan_dense_moe_layer_relu2(const cardan_shape* shape, int32_t B, const cardan_bf16* x,
                                 const cardan_dense_layer* layer, float* y, int32_t* topk_idx,
                                 float* topk_w, void* ws, size_t ws_bytes, hipStream_t stream);

/* RMS normalisation between stacked layers: x_next[t][h] =
 * bf16_rne(y[t][h] / sqrt(mean_h y[t][h]^2 + eps)), no learned scale.
 * y: [B][H] float32, x_next: [B][H] bf16. Needs no workspace. */
int cardan_rmsnorm_bf16(int32_t B, int32_t H, const float* y, float eps,
                        cardan_bf16* x_next, hipStream_t stream);

/* ---- training: the feed-forward block and the distillation loss -----------
 * The second stage of fitting a compressed layer (paper Sec. 3.3): a student
 * layer in dense bf16 form runs forward and backward over rows of any number,
 * and its logits are trained against a teacher's kept top logits, Eq. (3).
 * Conventions as above, except: the workspace of the feed-forward calls needs
 * no zero fill and holds nothing between calls (two calls that may overlap in
 * time, two captured graphs among them, need one each); the loss needs none.
 * Outputs must not overlap inputs or one another, except as said. No workgroup
 * of these kernels waits for another one. The stream's device must be the
 * current one. */

/* Shape of a feed-forward block: E matrix sets (experts) of hidden size H and
 * intermediate size I. H % 64 == 0, I % 32 == 0, both at most 2^20, H * I * 2
 * below 2^31, 1 <= E <= 1024; calls take 0 <= N <= 2^30 rows. */
typedef struct {
  int32_t H, I, E;
  int32_t act; /* CARDAN_FFN_SILU_GLU or CARDAN_FFN_RELU2_UP */
} cardan_ffn_shape;

enum {
  CARDAN_FFN_SILU_GLU = 0, /* h = silu(x W_gate) * (x W_up)                  */
  CARDAN_FFN_RELU2_UP = 1  /* h = max(x W_up, 0)^2 (NaN stays NaN); W_gate is not read */
};

/* Dense bf16 weights (device pointers), laid out as in cardan_dense_layer. */
typedef struct {
  const cardan_bf16* W_gate; /* [E][H][I] */
  const cardan_bf16* W_up;   /* [E][H][I] */
  const cardan_bf16* W_down; /* [E][I][H] */
} cardan_ffn_weights;

/* Workspace bytes of cardan_ffn_forward and cardan_ffn_backward for up to N
 * rows of this shape (0 is possible). Host-only. */
int cardan_ffn_workspace_bytes(const cardan_ffn_shape* shape, int32_t N, size_t* out);

/* The experts' computation of paper Sec. 2.1 on dense weights, for rows
 * grouped by expert: rows offsets[e] <= n < offsets[e + 1] of x [N][H] bf16
 * go through matrix set e, y[n] = W_down[e]^T h[n] with h[n] as the
 * activation says, float32 accumulation, y [N][H] bf16. h enters the second
 * product in bf16.
 * offsets: [E + 1] int32 on the device, non-decreasing, within [0, N]; NULL
 * with E == 1 means all rows. Groups may be empty. Rows in no group are not
 * read, and theirs of y (and of the kept activations) are left as they were.
 * Offsets outside [0, N] or decreasing are cut to ranges inside the tensors
 * (memory-safe); the rows concerned are then unspecified.
 * gate, up: [N][I] float32, hidden: [N][I] bf16: the activations that
 * cardan_ffn_backward reads. All three NULL: none are kept (gate is always
 * NULL with CARDAN_FFN_RELU2_UP). N may be 0: nothing is launched. */
int cardan_ffn_forward(const cardan_ffn_shape* shape, int32_t N, const cardan_bf16* x,
                       const int32_t* offsets, const cardan_ffn_weights* weights, cardan_bf16* y,
                       float* gate, float* up, cardan_bf16* hidden, void* ws, size_t ws_bytes,
                       hipStream_t stream);

/* Gradients of cardan_ffn_forward for the upstream gradient dy [N][H] bf16,
 * from its inputs and the activations that it kept:
 *   dh = dy W_down^T;  du = dh silu(g), dg = dh u silu'(g)  (or du = 2 dh max(u, 0))
 *   dx = dg W_gate^T + du W_up^T;  dW_gate = x^T dg, dW_up = x^T du, dW_down = h^T dy
 * with float32 accumulation; dg and du enter the products in bf16. dx [N][H]
 * bf16 or NULL; dW_gate and dW_up ([E][H][I] bf16, both or neither; dW_gate
 * NULL with CARDAN_FFN_RELU2_UP) or NULL; dW_down [E][I][H] bf16 or NULL: a
 * NULL output is not computed, one at least is required. Weight gradients are
 * written whole (zero for a group without rows), not accumulated. */
int cardan_ffn_backward(const cardan_ffn_shape* shape, int32_t N, const cardan_bf16* dy,
                        const cardan_bf16* x, const int32_t* offsets,
                        const cardan_ffn_weights* weights, const float* gate, const float* up,
                        const cardan_bf16* hidden, cardan_bf16* dx, cardan_bf16* dW_gate,
                        cardan_bf16* dW_up, cardan_bf16* dW_down, void* ws, size_t ws_bytes,
                        hipStream_t stream);

enum {
  CARDAN_LOGITS_BF16 = 0,
  CARDAN_LOGITS_F32 = 1,
  CARDAN_LOGITS_F64 = 2, /* routing calls alone */
  /* added to either: logits, teacher, ids, loss and dlogits need only start on
   * a multiple of their own elements' size (a slice of rows of odd length) */
  CARDAN_LOGITS_ANY_START = 16
};

/* Distillation loss of paper Sec. 3.3, Eq. (3), per row, with its gradient:
 * student logits s over V vocabulary entries (row n at logits + n * ld, type
 * `logits_type`), a teacher's K kept logits t_j at entries i_j
 * (teacher [N][K] float32, ids [N][K] int32), temperature T:
 *   kd = T^2 sum_j p_j (log p_j - log q_{i_j}),  p = softmax_j(t / T),
 *        q = softmax(s / T) over all V entries;
 *   ce = -log softmax(s)[label].
 * loss [N][2] float32 receives kd and ce. dlogits (type of the logits, row
 * stride dld; NULL: not computed) receives the gradient of
 * sum_n row_weight[n] (kd_n + ce_weight * ce_n), rounded once; it may be the
 * logits' own memory (dlogits == logits and dld == ld), and must not overlap
 * them otherwise. row_weight: [N] float32, NULL for ones.
 * An id outside [0, V), or one whose kept logit is -inf, is no entry (the
 * teacher's distribution is over the others; a row without any has kd = 0); a label outside [0, V) is none (ce =
 * 0); labels may be NULL. A row with neither gets zero loss and gradient and
 * its logits are not looked at. An entry named twice counts with both its
 * probabilities. -inf logits have probability 0 (a row of nothing else has no
 * softmax and gives NaN); NaN or +inf among a row's
 * logits give that row NaN; among the kept logits of its entries they give NaN
 * in kd and in the gradient at those entries. Values between V and the row strides are neither
 * read nor written.
 * 0 <= N <= 2^30, 1 <= V <= 2^30, 0 <= K <= 1024 (teacher and ids may be NULL
 * at K == 0), V <= ld, dld <= 2^40, 2^-16 <= T <= 2^16, ce_weight finite. */
int cardan_distill_loss(int32_t N, int32_t V, int32_t K, int32_t logits_type, const void* logits,
                        int64_t ld, const float* teacher, const int32_t* ids,
                        const int32_t* labels, float temperature, float ce_weight,
                        const float* row_weight, float* loss, void* dlogits, int64_t dld,
                        hipStream_t stream);

/* ---- training: the router, rows to their experts and back, the optimizer ---
 * What a routed layer of any number of rows has around its feed-forward block
 * (paper Sec. 2.1, Sec. 3.3): the routing whose places and offsets
 * cardan_ffn_forward's rows follow, with its gradient; the copies of the rows
 * and their weighted sums, with theirs; and the step that the gradients go
 * into. Conventions as for the training calls above, except that every pointer
 * but the workspace's need only start on a multiple of its own elements' size. */

enum { CARDAN_SCORE_SOFTMAX = 0, CARDAN_SCORE_SIGMOID = 1 };

/* How rows choose among E experts. 1 <= E <= 1024, 1 <= top_k <= min(E, 32),
 * 1 <= groups <= 64 dividing E, top_groups * (E / groups) >= top_k, group_best
 * 1 or 2 and at most E / groups, scale finite. groups = top_groups = group_best
 * = 1: no groups. */
typedef struct {
  int32_t E, top_k;
  int32_t score;      /* CARDAN_SCORE_SOFTMAX or CARDAN_SCORE_SIGMOID         */
  int32_t renorm;     /* 1: weights are divided by the sum of the kept scores */
  int32_t groups;     /* groups of E / groups consecutive experts             */
  int32_t top_groups; /* groups that a row may choose from                    */
  int32_t group_best; /* a group counts by its best (1) or best two (2)       */
  float scale;        /* factor of every weight                               */
} cardan_routing;

/* Workspace bytes of cardan_route_rows with places for up to N rows (0 for
 * few rows). No zero fill is needed, nothing is kept between calls. Host-only. */
int cardan_route_rows_workspace_bytes(const cardan_routing* routing, int32_t N, size_t* out);

/* Routing of N rows of logits z (row n at logits + n * ld; bf16, float32 or
 * float64). Scores s_e = softmax(z)_e over all E or sigmoid(z_e). The selection
 * goes by v_e = s_e + bias_e in float64 (bias: [E] float32) where there is a bias,
 * without one (NULL) by z_e, in the scores' order. A group counts by its best v
 * or the sum of its best two (of scores, with or without bias); of the top_groups best
 * groups (ties to the lower index) the top_k largest v are kept, descending,
 * exact ties to the lower index. weight_j = scale * s_j, divided by the sum of
 * the kept s with renorm; the bias is in no weight. With softmax, renorm, no
 * bias and no groups this is cardan_route_topk's routing.
 * idx [N][top_k] int32, weight [N][top_k] float32.
 * A logit of -inf (or a v of -inf) is an expert that is not there, whatever its
 * bias; where fewer than top_k are left (a padding row is one of -inf alone) the rest of idx is
 * -1 with weight 0. Weights below 2^-126 may be rounded to 0. A NaN among a row's logits or v is never selected and makes
 * the row's weights NaN; +inf makes a softmax row's weights NaN.
 * place [N][top_k] and offsets [E + 1] (both or neither NULL): the (row,
 * selection) pairs of an expert e are rows offsets[e] <= p < offsets[e + 1] of
 * the array grouped by expert, in their order, place their p; -1 where idx is.
 * ws is read with places alone. N * top_k below 2^31; N may be 0 (offsets are
 * zero then). Rows up to 2^40 elements apart. */
int cardan_route_rows(const cardan_routing* routing, int32_t N, int32_t logits_type, const void* logits, int64_t ld,
                      const float* bias, int32_t* idx, float* weight, int32_t* place, int32_t* offsets, void* ws,
                      size_t ws_bytes, hipStream_t stream);

/* Gradient of the logits for the gradient dweight [N][top_k] of
 * cardan_route_rows's weights at the experts idx that it chose (the selection
 * itself has none): with w the weights before scale and d = scale * dweight,
 *   renorm:  dz_j = w_j (d_j - sum_i w_i d_i), times (1 - s_j) with sigmoid
 *   sigmoid: dz_j = s_j (1 - s_j) d_j
 *   softmax: dz_e = s_e (d_e [e chosen] - sum_i s_i d_i) for every expert
 * in the logits' type, rounded once, written whole (zero at other experts).
 * dlogits may be the logits' own memory (dld == ld), and must not overlap them
 * otherwise. idx outside [0, E): no expert, its dweight is not looked at. An
 * expert named twice in a row gets one of its gradients. */
int cardan_route_rows_backward(const cardan_routing* routing, int32_t N, int32_t logits_type, const void* logits,
                               int64_t ld, const int32_t* idx, const float* dweight, void* dlogits, int64_t dld,
                               hipStream_t stream);

/* xe[place[n][j]] = x[n] for the k places of every row: x [N][H] bf16, place
 * [N][k] int32, xe [M][H] bf16. Places outside [0, M) are none; rows of xe that
 * no place names are left as they were. A row named twice is unspecified: any
 * mix of the two, not the same in every call. 1 <= k <= 32, 1 <= H <= 2^20. The
 * gradient is cardan_combine_rows without weights. */
int cardan_dispatch_rows(int32_t N, int32_t k, int32_t H, int32_t M, const cardan_bf16* x, const int32_t* place,
                         cardan_bf16* xe, hipStream_t stream);

/* y[n] = sum_j weight[n][j] * ye[place[n][j]] in float32 in the order of j,
 * rounded once to y's type (CARDAN_LOGITS_BF16 or _F32): ye [M][H] bf16, weight
 * [N][k] float32 or NULL for ones, y [N][H]. Places outside [0, M) add nothing
 * (their weights are not looked at); a row without any is zero. */
int cardan_combine_rows(int32_t N, int32_t k, int32_t H, int32_t M, const cardan_bf16* ye, const int32_t* place,
                        const float* weight, int32_t y_type, void* y, hipStream_t stream);

/* Gradients of cardan_combine_rows for dy [N][H] (bf16 or float32):
 *   dye[place[n][j]] = weight[n][j] * dy[n]   (bf16; rows without a place stay)
 *   dweight[n][j] = <dy[n], ye[place[n][j]]>  (float32; 0 without a place)
 * dye or dweight may be NULL (not computed; ye is read for dweight alone). A
 * row of dye named twice is unspecified: any mix of the two, not the same in
 * every call (dweight is not concerned). */
int cardan_combine_rows_backward(int32_t N, int32_t k, int32_t H, int32_t M, int32_t dy_type, const void* dy,
                                 const cardan_bf16* ye, const int32_t* place, const float* weight, cardan_bf16* dye,
                                 float* dweight, hipStream_t stream);

/* One tensor of an optimizer step (device pointers). n values each; with
 * 8-bit moments m holds e4m3 and v e5m2 values, and each has a float32 scale
 * for every 256 consecutive values ([ceil(n / 256)]). Zeros are the state
 * before the first step. */
typedef struct {
  void* param;        /* weights, updated                                     */
  const void* grad;
  void* m;            /* first moment, updated                                */
  void* v;            /* second moment, updated                               */
  float* m_scale;     /* 8-bit moments alone                                  */
  float* v_scale;
  cardan_bf16* copy;  /* receives float32 weights rounded to bf16, or NULL    */
  int64_t n;          /* values, 0 to 2^34                                    */
} cardan_adamw_tensor;

typedef struct {
  int32_t param_type;          /* CARDAN_LOGITS_BF16 or _F32, of all tensors  */
  int32_t grad_type;           /* likewise                                    */
  int32_t state_bits;          /* 32 (float32 moments) or 8                   */
  int32_t step;                /* t >= 1, unless step_device                  */
  double lr, beta1, beta2, eps, weight_decay;
  const int32_t* step_device;  /* t on the device (below 1 counts as 1), or NULL */
  const float* lr_device;      /* lr on the device, or NULL                   */
  const float* grad_scale;     /* factor of every gradient, on the device, or NULL (1) */
} cardan_adamw;

/* AdamW over `count` tensors (`tensors` is a host array; up to 40 share a
 * launch), for value p with gradient g (times grad_scale) at step t:
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   p = p - lr weight_decay p - lr m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps)
 * in float32. 8-bit moments enter the update as computed and are stored
 * rounded, with a scale of the largest size of their 256 over 448 (m) or
 * 57344 (v); these roundings, and those of bf16 weights, are dithered by a mix
 * of a value's place in its tensor and t (right in the mean; the same arguments
 * give the same result). Copies are rounded to nearest. A gradient that is not
 * finite goes on into its weight and moments; with 8-bit moments into those of
 * its 256 values. eps = 0 gives NaN where a gradient has always been 0. With
 * step_device and lr_device a captured call follows both.
 * Tensors must not overlap one another. */
int cardan_adamw_step(const cardan_adamw* config, int32_t count, const cardan_adamw_tensor* tensors,
                      hipStream_t stream);

/* Kernel timing for measurement. cardan_profile_begin(n) makes the next n
 * calls launch each kernel with a HIP start/stop event pair recorded by the
 * dispatch itself (hipExtLaunchKernel), on the call's stream, so the pair
 * brackets the kernel's execution; cardan_profile_end() waits for those
 * events and writes, per
 * kernel kind, the summed milliseconds and the launch count (arrays of
 * length CARDAN_PROFILE_KINDS, ordered as the enum below). A layer call runs
 * the routing kernel (routing, shared projections, grouping) and then the
 * expert kernel (gate/up, down, combine). Host-global state: not
 * thread-safe, not for use under graph capture. */
enum {
  CARDAN_KERNEL_ROUTE = 0,    /* router, top-k, gating, grouping, z = U^T x */
  CARDAN_KERNEL_EXPERT = 1,   /* gate/up, down, weighted combine            */
  CARDAN_KERNEL_RMSNORM = 2,
  CARDAN_PROFILE_KINDS = 3
};
int cardan_profile_begin(int32_t max_calls);
int cardan_profile_end(float* ms_per_kind, int32_t* launches_per_kind);

#ifdef __cplusplus
}
#endif

#endif /* CARDAN_H */
