/*
 * pcmoe_ext.h — calls around the expert layer of pcmoe.h: gated routing (softmax or sigmoid scores, balance bias, limited
 * expert groups) and its adjoint, 8-bit checkpoints of the activations that a forward saves, and experts with 4-bit weights.
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

#ifdef __cplusplus
}
#endif

#endif /* PCMOE_EXT_H */
