// Launchers of the gated routing, the 4-bit experts and the 8-bit activation checkpoints (private to the library).
#pragma once
#include "pcmoe_internal.h"
#include "../../include/pcmoe_ext.h"

namespace pcmoe {

// Gated routing (router.hip). Workspace of the adjoint: route_bwd_ws_bytes.
hipError_t launch_route_gated(const moe_desc& d, const moe_gate& g, const void* x, const void* wr, const float* bias,
                              int bias_groups, const float* select_bias, float* logits, int32_t* idx, float* w,
                              hipStream_t s);
hipError_t launch_route_gated_bwd(const moe_desc& d, const moe_gate& g, const void* x, const float* logits,
                                  const int32_t* idx, const float* w, const float* dgate, float* dlogits, float* dwr,
                                  void* ws, hipStream_t s);

// 8-bit checkpoints of the saved activations (checkpoint.hip).
size_t ffn_ckpt_bytes(const moe_desc& d);
hipError_t launch_ffn_checkpoint(const moe_desc& d, const int32_t* offsets, const void* saved, void* ckpt,
                                 hipStream_t s);
hipError_t launch_ffn_restore(const moe_desc& d, const int32_t* offsets, const void* ckpt, void* saved, hipStream_t s);

// 4-bit weights (experts_q4.hip): codes and scales of one projection of all experts.
struct Q4Weights {
  const void* codes;
  const void* scales;
};
size_t ffn_q4_ws_bytes(const moe_desc& d);
hipError_t launch_q4_pack(int n, int rows, int cols, int group, int dtype, const void* w, void* codes, void* scales,
                          hipStream_t s);
hipError_t launch_q4_unpack(int n, int rows, int cols, int group, int dtype, const void* codes, const void* scales,
                            void* w, hipStream_t s);
hipError_t launch_ffn_q4(const moe_desc& d, int group, const void* x, const void* xp, const int32_t* offsets,
                         const Q4Weights& gate, const Q4Weights& up, const Q4Weights& down, void* yp, void* ws,
                         hipStream_t s);

}  // namespace pcmoe
