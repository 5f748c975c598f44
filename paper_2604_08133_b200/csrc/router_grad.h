// Launchers of the router's gradients (router_grad.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "allocmoe.h"

// Bytes of workspace for balance_loss and gate_backward with this shape and up to n_seq sequences.
size_t router_workspace_bytes(const moe_shape* s, int32_t n_seq);

moe_status launch_balance_loss(const moe_shape* s, const float* scores, const int32_t* topk_idx, const int32_t* n_sel,
                               const int32_t* seq_offsets, int n_seq, float alpha, int32_t* counts, float* coef,
                               float* loss, int32_t* dev_status, void* ws, cudaStream_t stream);

struct GateBackwardArgs {
  const moe_shape* s;
  const uint16_t* x;
  const uint16_t* W_gate;
  const float* scores;
  const int32_t* topk_idx;
  const int32_t* n_sel;
  const float* d_topk_score;
  const float* coef;
  const int32_t* seq_offsets;
  int n_seq;
  float* d_logits;
  uint16_t* dx;
  float* dW;
  float* d_bias;
  int32_t* dev_status;
  void* ws;
  cudaStream_t stream;
};
moe_status launch_gate_backward(const GateBackwardArgs& a);

moe_status launch_combine_backward(const moe_shape* s, const uint16_t* d_out, const uint16_t* y_perm,
                                   const int32_t* pair_pos, const float* topk_score, const int32_t* n_sel,
                                   int64_t budget, float* d_topk_score, uint16_t* d_y_perm, cudaStream_t stream);
