// Launcher of the projections with low-rank adapters (adapter.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "allocmoe.h"

struct AdapterArgs {
  int T = 0, K = 0, M = 0, n_adapters = 0, rank = 0;
  int k_per_sub = 0;     // > 0: W is [K / k_per_sub][M][k_per_sub], the sub-experts' W2 one behind the other
  int swiglu_rows = 0;   // I > 0: W is [M / I][2I][K], y = silu(u1) * u3; B has the same 2M rows as W
  const uint16_t* x = nullptr;
  const uint16_t* W = nullptr;
  const uint16_t* A = nullptr;
  const uint16_t* B = nullptr;
  const float* scale = nullptr;
  const int32_t* adapter_id = nullptr;
  uint16_t* y = nullptr;
  int32_t* dev_status = nullptr;
  void* ws = nullptr;
  cudaStream_t stream = nullptr;
};

size_t adapter_workspace_bytes(int T, int rank);
moe_status launch_adapter_linear(const AdapterArgs& a);
