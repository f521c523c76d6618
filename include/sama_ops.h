/*
 * sama_ops.h -- op-level entry points of libsama: the individual kernels of the hot path, exposed for
 * per-kernel parity tests and roofline measurements.  Same conventions as sama.h: DEVICE pointers, work is
 * enqueued on the given hipStream_t (NULL = default stream) and not waited for, no allocation.
 */
#ifndef SAMA_OPS_H
#define SAMA_OPS_H

#include <stddef.h>
#include <stdint.h>
#include "sama.h"

#ifdef __cplusplus
extern "C" {
#endif

/* C[M x N] = A . (B + B2) on the bf16 matrix cores with fp32 accumulation: the contraction behind every linear
 * layer of the base learner (forward X W^T, dgrad dY W, wgrad dY^T X; Sec. 3.3 counts these passes).
 * a_trans = 0: A stored [M][K] (lda >= K); 1: stored [K][M] (lda >= M).
 * b_trans = 1: B stored [N][K] (ldb >= K), i.e. a weight matrix [out x in] used forward; 0: stored [K][N].
 * B2: optional second bf16 term of the weight (the low half of a two-term split), same storage as B, or NULL.
 * bias: optional fp32 [N] added to every row.  Outputs: C32 (fp32) and/or C16 (bf16), row stride ldc; either may
 * be NULL.  Requirements: K % 64 == 0, M % 8 == 0, N % 8 == 0, lda/ldb % 8 == 0, ldc % 4 == 0, 16-byte aligned
 * pointers.  Returns SAMA_EINVAL otherwise (nothing is launched). */
sama_status sama_op_gemm_bf16(const void* A, int64_t lda, int32_t a_trans, const void* B, const void* B2, int64_t ldb,
                              int32_t b_trans, int32_t M, int32_t N, int32_t K, const float* bias, float* C32, void* C16,
                              int64_t ldc, void* hip_stream);

/* `count` (1..4) independent contractions of the form above in ONE launch: the + and the - pass of Eq. 5 stacked, or the
 * four weight gradients of an encoder layer.  Every array is a HOST array of `count` entries; A[k], B[k], B2[k], C32[k]
 * are DEVICE pointers (B2 either given for every problem or NULL itself); operands are dense (lda = K or M, ldb = K
 * or N, ldc = N as the storage flags imply).  The problems share a_trans / b_trans; shapes may differ.  Same
 * requirements and error behaviour as sama_op_gemm_bf16. */
sama_status sama_op_gemm_bf16_batch(int32_t count, const void* const* A, const void* const* B, const void* const* B2,
                                    float* const* C32, const int32_t* M, const int32_t* N, const int32_t* K,
                                    int32_t a_trans, int32_t b_trans, void* hip_stream);

/* For tests (the encoder launches the kernels itself): the two GELU epilogues of the encoder's FFN on a dense hi + lo
 * contraction p = A . (B + B2).  With aux16 = NULL the forward form, C32 = gelu(bf16(p)) and pre16 = bf16(p); with aux16
 * (bf16 [M x N]) the backward form, C32 = p * gelu'(aux16), b_trans as above.  table: DEVICE scratch of
 * sama_op_gelu_table_bytes() bytes, 16-byte aligned, filled by the call. */
size_t sama_op_gelu_table_bytes(void);
sama_status sama_op_gemm_bf16_gelu(const void* A, const void* B, const void* B2, int32_t b_trans, int32_t M, int32_t N, int32_t K,
                                   const void* aux16, void* pre16, float* C32, void* table, void* hip_stream);

/* For tests: the residual epilogue of the encoder's hi + lo products, C32 = A . (B + B2)^T + bias + r, `count` (1 or 2) stacked passes of M rows
 * (A, x and C32 [count * M] rows; B [N x K] shared, B2 [count][N x K]).  params: [3][N] bias, gain and shift; with v ([3][N]) and eps (DEVICE
 * scalar), which go together, params + eps v in the first pass and params - eps v in the second.  stats NULL: r = x.  Else r is the LayerNorm's
 * output gain (x - mean) rstd + shift, stats: [2][count * M] means, then reciprocal deviations.  rows: DEVICE count, or NULL: only the first *rows
 * (at least 1, at most M) rows of each pass are computed, as in a padded batch. */
sama_status sama_op_gemm_bf16_residual(int32_t count, const void* A, const void* B, const void* B2, int32_t M, int32_t N, int32_t K,
                                       const float* params, const float* v, const float* eps, const float* x, const float* stats,
                                       float* C32, const int32_t* rows, void* hip_stream);

/* Base solver update, Adam form (Sec. 2; Kingma & Ba Alg. 1 with bias correction at step t >= 1), over n fp32
 * elements in place; theta16 (bf16 [n16], n16 <= n) receives the rounded leading part of theta, or NULL.  With
 * weight_decay != 0 the L2 term is added in front of the solver and g is overwritten with g + weight_decay * theta
 * (the gradient the solver was given, which the adaptation of Eq. 4 needs); with 0 g is only read. */
sama_status sama_op_adam(float* g, float* m, float* v, float* theta, void* theta16, int64_t n, int64_t n16,
                         int64_t t, float lr, float beta1, float beta2, float eps, float weight_decay, void* hip_stream);

/* Adaptation fused with the step size (Eq. 4-5, App. C): vdir = (du_adam/dg) . gmeta from the post-update moments at
 * step t, then scalars[0] = alpha / ||vdir||_2, scalars[1] = ||vdir||_2, status[0] = 1 if the norm is zero or not
 * finite (else 0).  partial: DEVICE scratch of 65536 doubles. */
sama_status sama_op_adapt_norm(const float* g, const float* m, const float* v, const float* gmeta, float* vdir,
                               double* partial, int64_t n, int64_t t, float lr, float beta1, float beta2, float eps,
                               float alpha, float* scalars, int64_t* status, void* hip_stream);

/* sama_op_adapt_norm for callers that cannot allocate or pass device scratch: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  Same arguments without `partial`, same results bit for bit: the
 * partial sums live in a 512 KB array inside the library's device image (one copy per GPU, held until the process
 * ends) whose address is resolved once per device at the first call there.  The call allocates nothing.  n must not
 * exceed SAMA_OP_STATIC_MAX_N; a larger n returns SAMA_EINVAL, launches nothing, and sama_op_last_error() says why.
 * Every call on a GPU shares that GPU's array: calls that overlap in time on one GPU (different streams or threads)
 * race on it -- serialise them, or use sama_op_adapt_norm with separate scratch buffers.  Nothing in the array needs
 * clearing between calls (each call overwrites the entries it reads). */
#define SAMA_OP_STATIC_MAX_N ((int64_t)1 << 29)
sama_status sama_op_adapt_norm_static(const float* g, const float* m, const float* v, const float* gmeta, float* vdir,
                                      int64_t n, int64_t t, float lr, float beta1, float beta2, float eps, float alpha,
                                      float* scalars, int64_t* status, void* hip_stream);
/* Text of the last error of an op-level call on this thread (HOST string owned by the library, "" if none); set by
 * sama_op_adapt_norm_static and the calls of a token model's step and sequences below. */
const char* sama_op_last_error(void);

/* Low halves of theta +- eps v against the bf16 working copy (Eq. 5): lo_p/lo_m[k] = bf16((theta[k] +- eps v[k]) -
 * float(bf16(theta[k]))), eps read from DEVICE eps_ptr. */
sama_status sama_op_perturb_lo(const float* theta, const float* vdir, const float* eps_ptr, void* lo_p, void* lo_m,
                               int64_t n16, void* hip_stream);

/* theta <- theta - eps v (end of Sec. 3.2), refreshing theta16 like sama_op_adam. */
sama_status sama_op_nudge(float* theta, const float* vdir, const float* eps_ptr, void* theta16, int64_t n, int64_t n16,
                          void* hip_stream);

/* ---- Operators of a token model's base step beyond the encoder's own: a scaled embedding, clipped gradients, and a gated
 * feed-forward block.
 * Types are SAMA_DTYPE_*; fp32 and bf16 may be mixed where a type is given for each side.  Strides (ld*) are in values, at least the row's length.
 * Any length, alignment (of a value) and stride is accepted, but for the bf16 block, see there; rows whose length, start and stride are multiples of 16 bytes are moved in
 * pieces of that size.  Sums are held in 32 bits or more, in a fixed order: the same call gives the same bits.  Workspaces need 256-byte
 * alignment and nothing in them beforehand; calls that overlap in time need one each.  Outputs must not overlap inputs, one another or the
 * workspace.  An argument that is refused gives SAMA_EINVAL, launches nothing, and sama_op_last_error() says which. */

/* out[i][:] = scale * table[id_i][:] for n tokens (table [V x d]).  Ids outside [0, V) are clamped into it, as everywhere in this
 * library; pad_id >= 0: the rows of that id (before clamping) are zero whatever the table holds there, -1: there is no such id. */
sama_status sama_op_embedding(const void* table, int32_t table_dtype, int64_t ld_table, const int32_t* ids, int64_t n, int32_t V, int32_t d,
                              float scale, int32_t pad_id, void* out, int32_t out_dtype, int64_t ld_out, void* hip_stream);

/* Its gradient: grad[v][:] = scale * sum over the i with id_i = v of dy[i][:], in ascending i (dy [n x d], grad [V x d]).  Padding contributes
 * nothing and its rows of dy are not read.  accumulate = 0: every row of grad is written, zeros where no token has the id; 1: the sums are
 * added to grad (a table that is also the output matrix), and rows without a token are left alone.  V is at most 2^30; n, up to
 * the next multiple of 128, times the pieces of a row (64 lanes' loads of 16 bytes each, of a value where rows do not consist of such) is below 2^30.  workspace: DEVICE,
 * sama_op_embedding_grad_bytes(n, V, d) bytes (0 for n below 0 or above 2^30, V or d below 1), which suffices for fewer tokens too. */
size_t sama_op_embedding_grad_bytes(int64_t n, int32_t V, int32_t d);
sama_status sama_op_embedding_grad(const void* dy, int32_t dy_dtype, int64_t ld_dy, const int32_t* ids, int64_t n, int32_t V, int32_t d,
                                   float scale, int32_t pad_id, int32_t accumulate, void* grad, int32_t grad_dtype, int64_t ld_grad,
                                   void* workspace, size_t workspace_bytes, void* hip_stream);

/* The global norm of `count` gradients and their clipping:  norm = sqrt(sum of all squares) (in 64 bits),
 * factor = min(1, max_norm / (norm + 1e-6)).  grads, counts, dtypes: HOST arrays of `count` DEVICE pointers, numbers of values and types.
 * out: DEVICE fp32 [sum of counts], receives factor * g of all tensors one after the other (the flat gradient of sama_op_adam), or NULL: the
 * gradients are scaled in place, and not touched where the factor is 1.  max_norm > 0; infinity gives the norm alone (out receives copies).
 * norm_out: DEVICE fp32 [2] = {norm, factor}, each rounded to fp32 (a finite norm beyond its range to infinity; what is applied is not the rounded factor
 * where that is below 2^-100, but one of all 24 bits).  status: DEVICE, or NULL: 1 if the norm is not finite, in which case the factor is 1, else 0.
 * workspace: DEVICE, sama_op_grad_clip_bytes() bytes.  The tensors must not overlap one another nor out. */
size_t sama_op_grad_clip_bytes(void);
sama_status sama_op_grad_clip(int64_t count, void* const* grads, const int64_t* counts, const int32_t* dtypes, float max_norm, float* out,
                              float* norm_out, int64_t* status, void* workspace, size_t workspace_bytes, void* hip_stream);

/* The gated feed-forward block for T tokens of width d with F hidden values:
 *     g = x Wg^T, u = x Wu^T, h = act(g) u, y = h w_out^T
 * x, y [T x d] with row strides ldx, ldy; w_in [2F x d], rows 0..F-1 = Wg, F..2F-1 = Wu; w_out [d x F]; hidden [T x F], receives h.  Matrices
 * without a stride are dense.  act: SAMA_ACT_SILU (g / (1 + exp(-g))) or SAMA_ACT_GELU (with the error function).
 * dtype SAMA_DTYPE_BF16: everything in bf16 with fp32 accumulation; h is rounded once, as y is.  d, F and the strides are multiples of 8 and
 * pointers 16-byte aligned.  SAMA_DTYPE_FP32: any d, F, stride and alignment of a value.  Strides at most 2^21, d and F at most 2^20, d F below 2^29
 * (fp32: 2^28).  T at most 2^22, 0 does nothing.  saved: DEVICE, sama_op_glu_ffn_saved_bytes() bytes, 16-byte aligned, receives what the backward call needs besides hidden (a layout
 * of the library's own), or NULL.  workspace: DEVICE, 256-byte aligned, sama_op_glu_ffn_bytes() bytes.  The size functions return 0 for sizes
 * that the calls refuse; a size for T tokens suffices for fewer.  What a token gets may depend in its last bits on how many tokens it comes
 * with; the same call gives the same bits. */
enum { SAMA_ACT_SILU = 0, SAMA_ACT_GELU = 1 };
size_t sama_op_glu_ffn_bytes(int64_t T, int32_t d, int32_t F, int32_t dtype);
size_t sama_op_glu_ffn_saved_bytes(int64_t T, int32_t F, int32_t dtype);
sama_status sama_op_glu_ffn(const void* x, int64_t ldx, const void* w_in, const void* w_out, int64_t T, int32_t d, int32_t F, int32_t act,
                            int32_t dtype, void* y, int64_t ldy, void* hidden, void* saved, void* workspace, size_t workspace_bytes,
                            void* hip_stream);

/* Its gradients, given dy [T x d] and the x, weights, hidden and saved of the forward call:
 *     dh = dy w_out, dg = dh u act'(g), du = dh act(g), dx = dg Wg + du Wu, dw_in = [dg; du]^T x, dw_out = dy^T h
 * dx [T x d] with row stride lddx in dtype; dw_in [2F x d] and dw_out [d x F], overwritten, in dw_dtype: dtype, or SAMA_DTYPE_FP32.  In bf16 dg and du
 * are rounded once before the products they enter.  With T = 0 the weights' gradients are zero.  workspace: sama_op_glu_ffn_grad_bytes() bytes. */
size_t sama_op_glu_ffn_grad_bytes(int64_t T, int32_t d, int32_t F, int32_t dtype);
sama_status sama_op_glu_ffn_grad(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w_in, const void* w_out, const void* hidden,
                                 const void* saved, int64_t T, int32_t d, int32_t F, int32_t act, int32_t dtype, void* dx, int64_t lddx,
                                 void* dw_in, void* dw_out, int32_t dw_dtype, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- Operators of a token model's sequences: rotary positions, attention within spans of keys, distillation from a teacher's top logits.
 * Types, streams, workspaces, overlap, order of sums and refusals as above.  [tokens][heads][width] tensors have a stride between tokens (ld) and one between heads (hs), in
 * values, each at least the width; the width is dense.  So the parts of a product's rows [T][(Hq + 2 Hk) D] can be taken in place, and [heads][tokens][width] as well. */

/* Rotary positions.  Of each head's D values the first R = 2 sum(sections) turn in pairs, pair i (i = 0 .. R/2 - 1) by phi = positions[a][t] base^(-2 i / R):
 *     (x, y) -> (x cos phi - y sin phi, x sin phi + y cos phi);  inverse = 1: by -phi, which is also the gradient.
 * neighbours = 0: pair i is values i and i + R/2; 1: values 2 i and 2 i + 1.  sections: HOST array [axes] of numbers of pairs: the first sections[0] turn by axis a = 0, the next
 * sections[1] by axis 1 and so on (time, height and width of a video; text has one axis).  positions: DEVICE int32 [axes][T], any value.  The other D - R values are copied.  Angles are
 * formed in 64 bits, off by 2^-46 of themselves or so; base is at least 1e-6 (below 1 an angle is up to |position| / base).  x and out [T][H][D] in dtype; out may be x itself, with the same strides.  axes 1 to 4, R 2 to 256, H D up to 2^20, T up to 2^23. */
sama_status sama_op_rotary(const void* x, int64_t ldx, int64_t hsx, int64_t T, int32_t H, int32_t D, int32_t dtype, const int32_t* positions, int32_t axes,
                           const int32_t* sections, double base, int32_t neighbours, int32_t inverse, void* out, int64_t ldo, int64_t hso, void* hip_stream);

/* Attention.  Query i of head h sees the keys begin <= j < end of its span (spans: DEVICE int32 [Tq][2], clipped to [0, Tk)) of key head h Hk / Hq:
 *     s_j = scale q_i . k_j;  with cap > 0: s_j = cap tanh(s_j / cap);  with slopes: s_j -= slopes[h] |at_i - j|
 *     p = softmax of s over those j,  out_i = sum_j p_j v_j,  lse_i = log sum_j exp(s_j)
 * A query that sees nothing has out = 0 and lse = minus infinity; one whose scores are all minus infinity has the same lse, but out is NaN, and its
 * gradients are not finite either.  Spans of packed documents come from sama_op_attention_spans; a cache per text, rows of padding,
 * windows or any other interval of keys for each query can be given as well, in any order.  Keys and values that a query does not see do not reach it, whatever they hold; a value that is not finite
 * reaches those that see it as one that is not finite, if not the same.
 * q, out [Tq][Hq][D], k, v [Tk][Hk][D]; Hk up to 2^20, Hq a multiple of it, at most 64 times; D a multiple of 8 up to 128; strides multiples of 16 bytes, ld at most 2^21, (Hq/Hk - 1) hs of q and dout
 * below 2^30 bytes; pointers 16-byte aligned; Tq Hq and Tk Hk up to 2^28.  at: DEVICE int32 [Tq], the place of each query among the keys, up to 2^30 to either
 * side of 0, or NULL: query i is beside key i (Tq = Tk).
 * slopes: DEVICE fp32 [Hq], or NULL; constants, they get no gradient; the bias is formed in 32 bits, off by up to 2^-22 slopes[h] |at_i - j|.  lse: DEVICE fp32 [Tq][Hq], natural logarithm, or NULL.  scale > 0; cap 0: none, or 1e-3 to 4096.
 * bf16: probabilities are rounded to bf16 before their product with v, sums are fp32; fp32: nothing is rounded.  workspace: sama_op_attention_bytes(), for these very sizes (0 for sizes that are refused). */
typedef struct { void* p; int64_t ld, hs; } sama_heads;
typedef struct {
  sama_heads q, k, v, out;
  const int32_t *spans, *at;
  const float* slopes;
  float* lse;
  int64_t Tq, Tk;
  int32_t Hq, Hk, D, dtype;
  float scale, cap;
  sama_heads dout, dq, dk, dv;   /* of the gradients */
} sama_attention;
size_t sama_op_attention_bytes(int64_t Tq, int64_t Tk, int32_t Hq, int32_t Hk, int32_t D, int32_t dtype);
sama_status sama_op_attention(const sama_attention* args, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Its gradients: dq, dk, dv, all overwritten, from dout, the inputs, out and lse of the forward call (HOST struct, the same arguments).  A query that sees nothing has dq = 0 and its rows of
 * q and dout reach nobody; keys that nobody sees have dk = dv = 0.  Key heads shared by several heads get the sum, in a fixed order.  bf16: probabilities and the scores' gradients
 * are rounded to bf16 before the products they enter, and sum_j p_j dp_j of a query that sees more than 8 keys is taken from out as it was rounded. */
size_t sama_op_attention_grad_bytes(int64_t Tq, int64_t Tk, int32_t Hq, int32_t Hk, int32_t D, int32_t dtype);
sama_status sama_op_attention_grad(const sama_attention* args, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Spans of T packed tokens: document n is the tokens offsets[n] <= t < offsets[n + 1] (DEVICE int32 [documents + 1], not decreasing; clipped to [0, T)), and a token sees its
 * document; causal = 1: of it only what is not behind the token, and the first prefix[n] tokens (DEVICE int32 [documents], or NULL: none).  Tokens outside every document see nothing. */
sama_status sama_op_attention_spans(const int32_t* offsets, int64_t documents, const int32_t* prefix, int32_t causal, int64_t T, int32_t* spans, void* hip_stream);

/* Distillation from a teacher's top logits, the loss of each token and its gradient.  Token i has student logits z [V] and up to K entries (ids[i][k], teacher[i][k]):
 *     p = softmax over its entries of teacher / temperature,  q = softmax over the vocabulary of z / temperature
 *     loss_i = temperature^2 sum_k p_k (log p_k - log q_{ids k}),   dz_ij = dloss_i temperature (q_j - sum over the k with ids k = j of p_k)
 * Entries with an id outside [0, V) or a logit of minus infinity are none, whatever else they hold; a token without entries has loss 0, gradient 0, and its logits are not read.  An id may be listed more than once.  With K = 1 and
 * temperature 1 this is the cross-entropy of a label.  q is formed in 32 bits: a loss is off by about temperature^2 2^-20, which at temperatures of hundreds may be all of a small one.  logits [T][V] in dtype with row stride ldz, any alignment; ids int32, teacher fp32 [T][K], dense; K 1 to 256; loss fp32 [T]; saved fp32 [T][2], for the gradient; temperature
 * 1e-4 to 1e4; V up to 2^30, T up to 2^22, 0 does nothing.  dlogits [T][V] in dtype, with stride lddz, may be logits themselves with the same stride; dloss fp32 [T]. */
sama_status sama_op_distill(const void* logits, int64_t ldz, int32_t dtype, int64_t T, int32_t V, const int32_t* ids, const float* teacher, int32_t K, float temperature,
                            float* loss, float* saved, void* hip_stream);
sama_status sama_op_distill_grad(const void* logits, int64_t ldz, int32_t dtype, int64_t T, int32_t V, const int32_t* ids, const float* teacher, int32_t K, float temperature,
                                 const float* dloss, const float* saved, void* dlogits, int64_t lddz, void* hip_stream);

/* Diagnostic switches, process-wide, for tests and profiling.  They take effect from the next launch and are not
 * thread-safe.
 *  - sama_dev_gemm_shape(id): every bf16 GEMM launch uses block tile `id`: 1..8 are the single-term tiles (a hi+lo
 *    problem then runs as one contraction over the concatenated operands, which rounds differently from the hi+lo
 *    tiles), 11..20 the hi+lo tiles (single-term problems ignore them, 20 is for K % 128 = 0); 0 = the heuristic (default).  Within a class
 *    every tile gives the same bits.
 *  - sama_dev_gemm_rows(choice): hi+lo products over the rows in use of a padded batch run in the launch that chooses its tile on the
 *    device, by `choice`: four bits for each sixteenth of the rows, the lowest for up to one, each 1 (256 x 192), 2 (256 x 128), 4 (128 x 96) or
 *    5 (128 x 64), anything else is SAMA_EINVAL; 0 = the heuristic (default).  No bit of a result depends on it.
 *  - sama_dev_gemm_counts(counts, 2): HOST counts since the last call: launches of that kernel for forward products and for input gradients.
 *  - sama_dev_glu_tile(t + 1000 p): the products of the gated feed-forward block use the t x t tile, t = 32, 64, 128 or 256, or 256 x 128 for
 *    t = 192 (fp32: 128 at most), and cut their contractions into p parts where these are long enough (t = 0 or p = 0: by the heuristic); 0 = the
 *    heuristic for both (default).  The order of the sums goes with p.  Anything else is SAMA_EINVAL and leaves the switch as it was.
 *  - sama_dev_side_stream(0): the encoder's backward passes keep every launch on the context's stream (a per-kernel profile
 *    wants one stream); 1 = default: weight gradients and optimizer slices run on the library's second stream where rows and
 *    layers are large enough for it; 2: they do for every size.  Any other value means 1.  A base step keeps its bits; a
 *    meta step adds the partial sums of ||v||^2 in another order.
 *  - sama_dev_side_sink(0): the optimizer and adaptation slices wait for the end of the backward pass instead of
 *    following each layer's gradients; 1 = default.  The same holds for its bits. */
void sama_dev_gemm_shape(int32_t id);
sama_status sama_dev_gemm_rows(uint64_t choice);
sama_status sama_dev_gemm_counts(int64_t* counts, int32_t n);
sama_status sama_dev_glu_tile(int32_t tile);
void sama_dev_side_stream(int32_t mode);
void sama_dev_side_sink(int32_t on);

#ifdef __cplusplus
}
#endif
#endif /* SAMA_OPS_H */
