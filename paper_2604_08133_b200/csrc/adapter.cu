// Projections with a low-rank adapter per request beside the shared weight:
//   v[t] = scale[a] x[t] A_a^T   (inner values, a = adapter_id[t])
//   y[t] = x[t] W^T + v[t] B_a^T
// and the same with SwiGLU on the pairs of output rows (the shared experts' first projection).
#include "adapter.h"
#include "common.cuh"

namespace allocmoe {

struct AdapterParams {
  int T, K, M, n_adapters, rank, k_per_sub, swiglu_rows;
  const uint16_t* x;
  const uint16_t* W;
  const uint16_t* A;
  const uint16_t* B;
  const float* scale;
  const int32_t* adapter_id;
  uint16_t* y;
  int32_t* dev_status;
  __nv_bfloat16* v;   // [T][rank]
};

// The adapter of token t, -1 for none.
DEV int adapter_of(const AdapterParams& p, int t) {
  const int a = __ldg(p.adapter_id + t);
  return a < 0 || a >= p.n_adapters ? -1 : a;
}

// Inner values: a CTA per token, a warp per row of A.
__global__ void __launch_bounds__(256)
adapter_inner_kernel(const AdapterParams p) {
  pdl_prologue_done();
  const int t = blockIdx.x, lane = threadIdx.x & 31;
  if (threadIdx.x == 0 && __ldg(p.adapter_id + t) >= p.n_adapters) set_dev_status(p.dev_status, MOE_ERR_ARG);
  const int a = adapter_of(p, t);
  if (a < 0) return;
  const float scale = __ldg(p.scale + a);
  const uint4* xr = reinterpret_cast<const uint4*>(p.x + (size_t)t * p.K);
  for (int r = threadIdx.x >> 5; r < p.rank; r += 8) {
    const uint4* ar = reinterpret_cast<const uint4*>(p.A + ((size_t)a * p.rank + r) * p.K);
    float acc = 0.f;
    for (int c = lane; c < p.K / 8; c += 32) {
      const uint4 xv = __ldg(xr + c), av = __ldg(ar + c);
      const uint32_t xu[4] = {xv.x, xv.y, xv.z, xv.w}, au[4] = {av.x, av.y, av.z, av.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        acc = fmaf(bf16_bits_to_float(xu[q] & 0xFFFFu), bf16_bits_to_float(au[q] & 0xFFFFu), acc);
        acc = fmaf(bf16_bits_to_float(xu[q] >> 16), bf16_bits_to_float(au[q] >> 16), acc);
      }
    }
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, d);
    if (lane == 0) p.v[(size_t)t * p.rank + r] = __float2bfloat16_rn(scale * acc);
  }
}

// Row `m` of the output's weight: with SwiGLU, output column m belongs to W1 row m % I of sub-expert m / I.
DEV size_t weight_row(const AdapterParams& p, int m, bool up) {
  if (p.swiglu_rows == 0) return m;
  const int s = m / p.swiglu_rows, i = m % p.swiglu_rows;
  return (size_t)s * 2 * p.swiglu_rows + (up ? p.swiglu_rows : 0) + i;
}

DEV float adapted_dot(const AdapterParams& p, int t, int m, bool up, int a, float base) {
  if (a < 0) return base;
  const size_t row = weight_row(p, m, up), rows = p.swiglu_rows > 0 ? 2 * (size_t)p.M : (size_t)p.M;
  float acc = base;
  for (int r = 0; r < p.rank; ++r)
    acc = fmaf(__bfloat162float(p.v[(size_t)t * p.rank + r]),
               bf16_bits_to_float((uint32_t)__ldg(p.B + ((size_t)a * rows + row) * p.rank + r)), acc);
  return acc;
}

// 32 tokens x 32 output columns a CTA, K in steps of 32 through shared memory.
__global__ void __launch_bounds__(256)
adapter_linear_kernel(const AdapterParams p) {
  __shared__ float xs[32][33], w1[32][33], w3[32][33];
  pdl_prologue_done();
  const int t0 = blockIdx.y * 32, m0 = blockIdx.x * 32;
  const int col = threadIdx.x & 31, row0 = (threadIdx.x >> 5) * 4;
  const bool glu = p.swiglu_rows > 0;
  float a1[4] = {0.f, 0.f, 0.f, 0.f}, a3[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < p.K; k0 += 32) {
    __syncthreads();
    for (int i = 0; i < 4; ++i) {
      const int r = row0 + i, k = k0 + col, t = t0 + r, m = m0 + r;
      const bool kk = k < p.K;
      xs[r][col] = kk && t < p.T ? bf16_bits_to_float((uint32_t)__ldg(p.x + (size_t)t * p.K + k)) : 0.f;
      w1[r][col] = w3[r][col] = 0.f;
      if (kk && m < p.M) {
        const size_t at = p.k_per_sub > 0
                              ? ((size_t)(k / p.k_per_sub) * p.M + m) * p.k_per_sub + k % p.k_per_sub
                              : weight_row(p, m, false) * p.K + k;
        w1[r][col] = bf16_bits_to_float((uint32_t)__ldg(p.W + at));
        if (glu) w3[r][col] = bf16_bits_to_float((uint32_t)__ldg(p.W + weight_row(p, m, true) * p.K + k));
      }
    }
    __syncthreads();
    for (int k = 0; k < 32; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a1[i] = fmaf(xs[row0 + i][k], w1[col][k], a1[i]);
        if (glu) a3[i] = fmaf(xs[row0 + i][k], w3[col][k], a3[i]);
      }
  }
  const int m = m0 + col;
  if (m >= p.M) return;
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + row0 + i;
    if (t >= p.T) continue;
    const int a = adapter_of(p, t);
    float v = adapted_dot(p, t, m, false, a, a1[i]);
    if (glu) v = v / (1.f + __expf(-v)) * adapted_dot(p, t, m, true, a, a3[i]);
    p.y[(size_t)t * p.M + m] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
  }
}

}  // namespace allocmoe

using namespace allocmoe;

size_t adapter_workspace_bytes(int T, int rank) { return (((size_t)T * rank * 2) + 255) & ~(size_t)255; }

moe_status launch_adapter_linear(const AdapterArgs& a) {
  AdapterParams p{};
  p.T = a.T;
  p.K = a.K;
  p.M = a.M;
  p.n_adapters = a.n_adapters;
  p.rank = a.rank;
  p.k_per_sub = a.k_per_sub;
  p.swiglu_rows = a.swiglu_rows;
  p.x = a.x;
  p.W = a.W;
  p.A = a.A;
  p.B = a.B;
  p.scale = a.scale;
  p.adapter_id = a.adapter_id;
  p.y = a.y;
  p.dev_status = a.dev_status;
  p.v = static_cast<__nv_bfloat16*>(a.ws);
  if (launch_dependent(adapter_inner_kernel, dim3((unsigned)a.T), dim3(256), 0, a.stream, 1, p) != cudaSuccess) return MOE_ERR_CUDA;
  const dim3 grid((unsigned)((a.M + 31) / 32), (unsigned)((a.T + 31) / 32));
  return launch_dependent(adapter_linear_kernel, grid, dim3(256), 0, a.stream, 1, p) == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}
