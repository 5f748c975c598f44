// Launchers of the calls for training the layer: ragged products and the experts' backward pass (grouped.cu), the norms
// around a block (block_norm.cu), the optimizer (adamw.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "allocmoe.h"

moe_status launch_grouped_gemm(const moe_grouped_shape* s, const uint16_t* x, const int32_t* offsets, const uint16_t* W, uint16_t* y,
                               int32_t* dev_status, cudaStream_t stream);
moe_status launch_grouped_gemm_dx(const moe_grouped_shape* s, const uint16_t* dy, const int32_t* offsets, const uint16_t* W, uint16_t* dx,
                                  int32_t* dev_status, cudaStream_t stream);
moe_status launch_grouped_gemm_dw(const moe_grouped_shape* s, const uint16_t* dy, const uint16_t* x, const int32_t* offsets, void* dW,
                                  int32_t* dev_status, cudaStream_t stream);

// E groups of S sub-experts each: routed experts have S 1, the shared experts are one group (E 1, no offsets).
struct FfnBackwardArgs {
  int E = 0, S = 1, H = 0, I = 0;
  int64_t rows = 0;                        // of the list
  const int32_t* offsets = nullptr;        // device [E+1]; nullptr with E 1: all rows
  const uint16_t* x = nullptr;             // the list's rows [rows, H]; with perm_token the tokens [T, H]
  const int32_t* perm_token = nullptr;
  int T = 0;
  uint16_t* x_rows = nullptr;              // [rows, H] scratch, for perm_token
  const uint16_t* W13 = nullptr;           // [E, S, 2I, H]
  const uint16_t* W2 = nullptr;            // [E, S, H, I]; S above 1 with E 1 alone
  const uint16_t* d_y = nullptr;           // [rows, H]
  uint16_t* h = nullptr;                   // [rows, S*I] scratch
  uint16_t* du = nullptr;                  // [rows, S*2I] scratch
  uint16_t* dx = nullptr;                  // optional outputs
  uint16_t* dW13 = nullptr;
  uint16_t* dW2 = nullptr;
  int32_t* dev_status = nullptr;
  cudaStream_t stream = nullptr;
};
moe_status launch_ffn_backward(const FfnBackwardArgs& a);

struct BlockNormArgs {
  const moe_norm_shape* s = nullptr;
  const uint16_t* r = nullptr;             // backward: r_out
  const uint16_t* y = nullptr;
  const float* w_post = nullptr;
  const uint16_t* gate = nullptr;
  const float* scale = nullptr;
  const float* w_pre = nullptr;
  uint16_t* r_out = nullptr;               // forward
  uint16_t* n_out = nullptr;
  const uint16_t* d_n = nullptr;           // backward
  const uint16_t* d_r_out = nullptr;
  uint16_t* d_r = nullptr;
  uint16_t* d_y = nullptr;
  uint16_t* d_gate = nullptr;
  float* dw_post = nullptr;
  float* dw_pre = nullptr;
  float* d_scale = nullptr;
  void* ws = nullptr;
  cudaStream_t stream = nullptr;
};
size_t block_norm_workspace_bytes(const moe_norm_shape* s);
moe_status launch_block_norm(const BlockNormArgs& a);
moe_status launch_block_norm_backward(const BlockNormArgs& a);

struct AdamwArgs {
  const moe_adamw_tensor* tensors = nullptr;   // host
  int count = 0;
  double beta1 = 0.0, beta2 = 0.0, eps = 0.0;
  const float* hyper = nullptr;
  const float* const* m32 = nullptr;           // states_read / states_write
  const float* const* v32 = nullptr;
  int32_t* dev_status = nullptr;
  cudaStream_t stream = nullptr;
};
bool adamw_chunks_ok(const moe_adamw_tensor* tensors, int count);
moe_status launch_adamw_step(const AdamwArgs& a);
moe_status launch_adamw_read(const AdamwArgs& a);
moe_status launch_adamw_write(const AdamwArgs& a);
