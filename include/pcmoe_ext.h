/*
 * pcmoe_ext.h — calls around the expert layer of pcmoe.h: gated routing (softmax or sigmoid scores, balance bias, limited
 * expert groups) and its adjoint, 8-bit checkpoints of the activations that a forward saves, experts with 4-bit weights and
 * experts in 8-bit integers, the norms, gate and residual between two layers with their adjoint, and updates of the experts'
 * matrices by their orthogonalised momentum.
 * Same library, same conventions: device pointers, 16-byte aligned tensors and 256-byte aligned workspaces (the bias vectors
 * only need 4-byte alignment), nothing allocated and nothing waited for, arguments checked before any launch, the statuses of
 * pcmoe.h. Routing reads its scores' definition, and the experts their row space, from there.
 */
#ifndef PCMOE_EXT_H
#define PCMOE_EXT_H

#include "pcmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How gated routing scores and selects. */
typedef enum { MOE_SCORE_SOFTMAX = 0, MOE_SCORE_SIGMOID = 1 } moe_score_kind;
typedef struct {
  int32_t score;        /* moe_score_kind */
  int32_t n_groups;     /* groups of n_experts / n_groups consecutive experts; divides n_experts, at most 64; 1: none */
  int32_t topk_groups;  /* groups open to a token, 1..n_groups */
  int32_t group_top;    /* a group's value: its largest choice value (1), or the sum of its two largest (2) */
  float scale;          /* factor of the gate weights, > 0, finite and not subnormal */
} moe_gate;
#define MOE_NO_EXPERT 0x7fffffff /* topk_idx of a slot that no expert fills */

/*
 * Gating with softmax or sigmoid scores, a balance bias and limited groups. With l = W_g h (+ logit_bias), formed as in
 * moe_route, s = softmax(l) or 1 / (1 + exp(-l)) and c = s + select_bias:
 *   - the topk_groups groups of largest value are open (all of them when n_groups = 1);
 *   - I = the k experts of the open groups with the largest c, in descending order;
 *   - w = scale * s[I] / sum s[I] (renormalize = 1) or scale * s[I]; the bias has no part in the weights.
 * s and c are formed in fp64 from the fp32 l; without select_bias the experts rank by l itself (the same order). Equal
 * values go to the lower index, experts and groups alike. An expert whose l or bias is NaN or -inf is never selected and
 * one whose l is has no part in the softmax; a group's value sums what selectable experts it has. Experts of l = +inf share
 * the softmax equally, as its limit. Slots left over get MOE_NO_EXPERT and weight 0: the other calls take them as slots
 * hosted elsewhere. Where all the selected s are 0 in fp64, renormalised weights are 0.
 *   select_bias [E] fp32 or NULL; logit_bias, bias_groups, the other arguments and their layouts: moe_route
 * Errors as above, and MOE_ERR_INVALID_ARGUMENT for a setting outside the ranges stated in moe_gate, group_top = 2 with
 * groups of one expert, or top_k > topk_groups * (E / n_groups); MOE_ERR_UNSUPPORTED for more than 64 groups.
 */
moe_status moe_route_gated(const moe_desc* desc, const moe_gate* gate, const void* x, const void* w_router,
                           const float* logit_bias, int32_t bias_groups, const float* select_bias, float* logits,
                           int32_t* topk_idx, float* topk_w, hipStream_t stream);

/*
 * Adjoint of moe_route_gated (selection has no gradient). With g = dgate, c = scale and w, s as returned and defined there:
 *   renormalize=1: dlogits[t, I_tj] = w_tj (g_tj - sum_j' w_tj' g_tj' / c), times (1 - s_tj) for sigmoid scores
 *   renormalize=0: sigmoid: dlogits[t, I_tj] = w_tj (1 - s_tj) g_tj;
 *                  softmax: dlogits[t, e] = s_te (c g_te - sum_e' s_te' c g_te'), g scattered onto E
 * and 0 elsewhere; slots of MOE_NO_EXPERT give nothing, whatever their dgate holds.
 *   dw_router = dlogits^T x and the other arguments: moe_route_bwd, whose conditions hold here too. logits is always needed.
 *   For bf16 x, dlogits is multiplied as three bf16 numbers that add up to it: an infinite x can give NaN in place of an
 *   infinity.
 */
moe_status moe_route_gated_bwd(const moe_desc* desc, const moe_gate* gate, const void* x, const float* logits,
                               const int32_t* topk_idx, const float* topk_w, const float* dgate, float* dlogits,
                               float* dw_router, void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * What moe_expert_ffn_fwd saved, kept in 8 bits until the backward: a layer then holds MOE_WS_FFN_CKPT bytes (about 2.06
 * per element of H) in place of MOE_WS_FFN_SAVED (6 in bf16, 12 in fp32), and one saved buffer serves all the layers.
 *   moe_ffn_checkpoint  reads saved after the forward and writes ckpt;
 *   moe_ffn_restore     writes saved for the moe_expert_ffn_bwd of the same call shape and offsets.
 * 32 consecutive columns of a row of G|U share a power of two 2^e, the smallest with max|v| <= 127 2^e (-126 <= e <= 121); a
 * value is restored as 2^e times rint(v / 2^e), ties to even, at most 127 either way, which no dtype rounds again.
 * Infinities and NaN are restored as NaN and do not count for e. H is restored as silu(G) U of the restored values.
 *   saved   G|U [R, 2f] dtype, at the next multiple of 256 bytes H [R, f] dtype, then the tile plan (opaque)
 *   ckpt    MOE_WS_FFN_CKPT bytes (opaque), 256-byte aligned as a workspace
 * Rows [offsets[local_count], T*k) are neither read nor written. One call's ckpt and saved must not overlap.
 */
moe_status moe_ffn_checkpoint(const moe_desc* desc, const int32_t* offsets, const void* saved, void* ckpt,
                              size_t ckpt_bytes, hipStream_t stream);
moe_status moe_ffn_restore(const moe_desc* desc, const int32_t* offsets, const void* ckpt, size_t ckpt_bytes,
                           void* saved, hipStream_t stream);

/*
 * 4-bit weights. A weight matrix [rows, cols] (rows out, cols in) is held as codes and scales: groups of `group` (32, 64
 * or 128) consecutive columns of a row share a bf16 scale, and a weight is scale * v with v one of 0, 0.5, 1, 1.5, 2, 3,
 * 4, 6 (code 0..7) or its negative (code + 8).
 *   codes   [n, rows/16, cols/128, q = 4, i = 16, s = 4, b = 4] bytes: row 16 rb + i; the low half of byte b is column
 *           128 cb + 32 s + 8 q + 2 b, the high half the next
 *   scales  [n, rows/16, cols/group, 16] bf16
 * moe_q4_pack makes them from n matrices w [n, rows, cols] of dtype: scale = bf16(max|w| * fp32(1/6)) of the group, code = the
 * nearest to w / scale, ties to the even code; a group with a NaN or an infinity gets a NaN scale. moe_q4_unpack writes
 * the weights that they stand for (in bf16 rounded once).
 * MOE_ERR_INVALID_ARGUMENT: n, rows or cols < 1, bad group or dtype, null or misaligned pointers; MOE_ERR_UNSUPPORTED: rows
 * not a multiple of 16, cols not one of 128, n * rows * cols >= 2^40.
 */
moe_status moe_q4_pack(int32_t n, int32_t rows, int32_t cols, int32_t group, int32_t dtype, const void* w, void* codes,
                       void* scales, hipStream_t stream);
moe_status moe_q4_unpack(int32_t n, int32_t rows, int32_t cols, int32_t group, int32_t dtype, const void* codes,
                         const void* scales, void* w, hipStream_t stream);

/*
 * moe_expert_ffn_fwd from 4-bit weights, for inference over few rows per expert (decoding, short prompts; nothing is saved
 * for a backward): H = silu(h W_gate^T) * (h W_up^T), O = H W_down^T for every hosted and every shared expert. Sums over
 * codes are held in fp32 and scaled in fp32. H is held in fp32, or for bf16 in two bf16 numbers, its rounding and the
 * rounding of the rest, so that a bf16 output is a sum rounded once. The order of the sums over K follows the shape of the
 * call: equal calls give equal bits, a row in a batch of another size can differ in its last bits.
 *   x, x_perm, offsets, y_perm   as for moe_expert_ffn_fwd
 *   gate_*, up_*   [local_count + n_shared] matrices [f, d], down_* [d, f], codes and scales as above, one group size
 *   ws      MOE_WS_FFN_Q4 bytes of scratch (H); calls that overlap on the GPU need their own
 */
moe_status moe_expert_ffn_q4(const moe_desc* desc, int32_t group, const void* x, const void* x_perm,
                             const int32_t* offsets, const void* gate_codes, const void* gate_scales,
                             const void* up_codes, const void* up_scales, const void* down_codes,
                             const void* down_scales, void* y_perm, void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * 8-bit rows. A row v of a matrix [rows, cols] is held as scale = fp32(m / 127), m = max|v|, and codes rint(127 v / m), ties
 * to even; a value stands for code * scale. A row of zeros has scale 0; a row with a NaN or an infinity has a NaN scale and
 * codes 0. For weights a row is an output channel.
 *   codes   [n, rows, cols] int8, scales [n, rows] fp32
 * moe_q8_pack makes them from n matrices w [n, rows, cols] of dtype; moe_q8_unpack writes the values that they stand for
 * (formed in fp32, in bf16 rounded again).
 * MOE_ERR_INVALID_ARGUMENT: n, rows or cols < 1, bad dtype, null or misaligned pointers; MOE_ERR_UNSUPPORTED: cols not a
 * multiple of 128, n * rows * cols >= 2^40.
 */
moe_status moe_q8_pack(int32_t n, int32_t rows, int32_t cols, int32_t dtype, const void* w, void* codes, void* scales,
                       hipStream_t stream);
moe_status moe_q8_unpack(int32_t n, int32_t rows, int32_t cols, int32_t dtype, const void* codes, const void* scales,
                         void* w, hipStream_t stream);

/*
 * moe_expert_ffn_fwd in 8-bit integers, for inference, prompts above all (nothing is saved for a backward). Rows of h and of
 * H are held in 8 bits as above, each with its own scale s; for every hosted and every shared expert
 *   G = s_h s_gate (h . gate), U = s_h s_up (h . up), H = silu(G) U, O = s_H s_down (H . down)
 * with sums over codes in 32-bit integers (exact), everything else in fp32, and O rounded once. A row's outputs do not depend
 * on the other rows of the call. A NaN or an infinity in a row of h, or a NaN scale of gate or up, makes the whole rows
 * of O that it reaches NaN.
 *   x, x_perm, offsets, y_perm   as for moe_expert_ffn_fwd
 *   gate_*, up_*   [local_count + n_shared] matrices [f, d], down_* [d, f], codes and scales as above
 *   ws      MOE_WS_FFN_Q8 bytes of scratch (codes of h and H, and H); calls that overlap on the GPU need their own
 * MOE_ERR_UNSUPPORTED for fp32 layers: an H next to the border between two codes would make outputs differ by far more than
 * fp32 allows.
 */
moe_status moe_expert_ffn_q8(const moe_desc* desc, const void* x, const void* x_perm, const int32_t* offsets,
                             const void* gate_codes, const void* gate_scales, const void* up_codes, const void* up_scales,
                             const void* down_codes, const void* down_scales, void* y_perm, void* ws, size_t ws_bytes,
                             hipStream_t stream);

/* Between two layers. */
typedef enum { MOE_NORM_NONE = 0, MOE_NORM_RMS = 1, MOE_NORM_LAYER = 2 } moe_norm_kind;
typedef struct {
  int32_t pre;           /* moe_norm_kind of the next block's input h */
  int32_t post;          /* ... and of the last block's output y */
  float eps;             /* > 0 and finite */
  float residual_scale;  /* alpha, finite */
  int32_t gate_groups;   /* rows of gate, dividing T: 1 a scale of the layer, T one for each token (any value without a gate) */
} moe_norm;

/*
 * What stands between two blocks of a stack, in one pass:
 *   r_t = alpha x_t + gamma_t * Npost(y_t),  h_t = Npre(r_t)
 * with gamma_t = gate[t / (T / gate_groups)] (1 without a gate) and
 *   RMS:   N(v) = v / sqrt(mean(v^2) + eps) * w
 *   LAYER: N(v) = (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps) * w
 *   NONE:  N(v) = v (no weight); with pre = NONE no h is written
 * h is formed from r before r is rounded. Before the first block y is NULL and h = Npre(x): r is x and is not written, and
 * there is no post norm, no gate, and alpha is 1.
 *   x, y    [T, d] dtype: the residual stream and the block's output (from moe_combine)
 *   w_post, w_pre [d] dtype or NULL (all ones); NULL where the norm is NONE
 *   gate    [gate_groups, d] dtype or NULL
 *   r, h    [T, d] dtype out; r may be x or y itself, h may be none of the inputs
 * The descriptor is checked as for the other calls; T, d_model and dtype of it are used. Sums over a row are held in fp64, means
 * in two fp32 parts: rows far from zero, and next to the end of the type's range, lose no digits.
 * MOE_ERR_INVALID_ARGUMENT for a setting outside the ranges stated in moe_norm, and for weights, a gate or outputs that the
 * setting has no place for.
 */
moe_status moe_residual_norm(const moe_desc* desc, const moe_norm* norm, const void* x, const void* y, const void* w_post,
                             const void* gate, const void* w_pre, void* r, void* h, hipStream_t stream);

/*
 * Adjoint of moe_residual_norm at (r, y), from the gradients dr of r (from the rest of the stack) and dh of h:
 *   g = dr + the gradient of r through h;  dx = alpha g;  dy = gamma * g back through Npost
 *   dw_pre = sum_t dh_t * r^_t, dw_post = sum_t gamma_t g_t * y^_t, dgate = sum over a gate row's tokens of g_t * Npost(y_t)
 * (^: normalised, before the weight). The norms' statistics are formed again from r and y, r as it was rounded. Sums over a row
 * are fp64 sums of those of 16 bytes of it, which are fp32 where gradients are multiplied; sums over tokens are fp32 and have a
 * fixed order: equal calls give equal bits.
 *   dr      [T, d] dtype, or NULL for zeros (the last block's r is used by nothing but h)
 *   dh      [T, d] dtype, NULL where pre is NONE
 *   y, r    [T, d] dtype: y NULL before the first block, where r is x; r may be NULL where pre is NONE, y where neither a
 *           post norm nor a gate needs it and dy is given
 *   dx, dy  [T, d] dtype out; dx may be dr or dh itself, dy may be y itself or dh; dy is NULL before the first block
 *   dw_post, dw_pre [d], dgate [gate_groups, d] fp32 out; NULL where there is no such weight or gate
 *   ws      MOE_WS_NORM_BWD bytes of scratch; calls that overlap on the GPU need their own
 */
moe_status moe_residual_norm_bwd(const moe_desc* desc, const moe_norm* norm, const void* dr, const void* dh, const void* y,
                                 const void* r, const void* w_post, const void* gate, const void* w_pre, void* dx, void* dy,
                                 float* dw_post, float* dgate, float* dw_pre, void* ws, size_t ws_bytes,
                                 hipStream_t stream);

/* Update by the orthogonalised momentum. */
typedef struct {
  float lr;            /* learning rate, > 0 */
  float momentum;      /* mu, in [0, 1) */
  float weight_decay;  /* decoupled decay factor, >= 0 (the parameter shrinks by lr * weight_decay) */
  float scale;         /* factor of the orthogonalised matrix, > 0; the same for gate, up and down */
  float eps;           /* added to the norm, > 0 */
  int32_t nesterov;    /* 1: u = g + mu m; 0: u = m */
  int32_t steps;       /* Newton-Schulz steps, 1..16 */
  float a, b, c;       /* their coefficients */
  int32_t precise;     /* 0: X and its products in fp16; 1: in two fp16 parts, at three times the operations */
} moe_muon;

/*
 * Another update of the expert parameters that ends the host's step in Alg. 6 (moe_expert_update): the momentum of every
 * weight matrix of every hosted and shared expert, made orthogonal by Newton-Schulz steps (as the Muon optimiser does):
 *   m <- mu m + g;  u = g + mu m or m;  X = u / (|u|_F + eps)
 *   steps times: A = X X^T, X <- a X + (b A + c A^2) X      (of a matrix with more rows than columns, of its transpose)
 * (steps may be taken together as one polynomial of A, which multiplies X once)
 *   p <- p (1 - lr weight_decay) - lr scale X
 * Norms are held in fp64, the momentum and all sums in fp32. X, A and a + b A + c A^2 are held in fp16 between products (11
 * bits, scaled by powers of two so that none overflows): X is off by some 2^-10 to 2^-8 of its size in the end, more where a few
 * directions of u are 20 times the others' size. With precise = 1 they are held in two fp16 parts each (22 bits), which leaves
 * X as exact as fp32 products do. A matrix whose u holds a NaN or an infinity becomes NaN, no other does.
 *   w_*, dw_*, master   as for moe_expert_update;  m  fp32 [P] momentum, updated in place
 *   ws   MOE_WS_UPDATE_MUON bytes of scratch, with precise = 1 MOE_WS_UPDATE_MUON_PRECISE bytes
 * MOE_ERR_INVALID_ARGUMENT for a setting outside the ranges stated in moe_muon; MOE_ERR_UNSUPPORTED for coefficients by which
 * a singular value of [0, 1] can pass 16, and for precise = 1 with d_model * d_ff >= 2^29. Calls that overlap on the same
 * parameters or workspace race.
 */
moe_status moe_expert_update_muon(const moe_desc* desc, const moe_muon* opt, void* w_gate, void* w_up, void* w_down,
                                  const void* dw_gate, const void* dw_up, const void* dw_down, float* master, float* m,
                                  void* ws, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PCMOE_EXT_H */
