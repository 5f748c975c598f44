// AdamW over many tensors in one launch, with moments in 32 or in 8 bits (formulas: allocmoe.h).
//
// Bound by memory: with an fp32 parameter, a bf16 gradient and a bf16 copy an element moves 28 bytes with 32-bit moments
// and 16 with 8-bit ones, for about 20 operations.  The list of tensors travels in the launch's own parameters (80 bytes an
// entry, up to 400), so nothing has to be laid out on the device before a step and a captured step is self-contained.  A CTA
// takes one chunk of kChunk elements of one tensor, found by a binary search over the chunks' prefix sums.
//
// A warp takes 256 consecutive elements at a time, which is also the block that shares a scale in 8 bits: lane l holds
// elements 4l .. 4l+3 and 128 + 4l .. 128 + 4l+3, so that every load of fp32 is 16 bytes a lane and contiguous over the warp
// with no more than 16-byte alignment, and a block's maximum is five shuffles.
//
// 190 M parameters with fp32 master, bf16 gradient and copy: 793 us with 32-bit moments, 6.7 TB/s; 551 us with 8-bit ones, 5.5 TB/s: loads one
// block ahead and three CTAs an SM took it from 790 to 615, packed products to 600, one division a block for scales and factors, codes through half
// precision and maxima by one instruction to 544, the look for an infinite v back to 551.  What is left is no longer instructions alone: roots that are approximate but for the neighbourhood
// of the codes' middles (the same bits) did not help.  Reading 8-bit moments back: 286 us, 6.7 TB/s; writing them 346.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"
#include "train.h"

namespace allocmoe {

constexpr int kAdamThreads = 256;
constexpr int kChunk = 4096;             // elements a CTA takes: two blocks of 256 a warp
constexpr int kBlock = 256;              // elements that share a scale
constexpr float kTopM = 448.f, kTopV = 1.9375f;
constexpr float kZeroBlock = 7.888609052210118e-31f;   // 2^-100
constexpr float kMostFinite = 3.402823466e38f, kMostRoot = 1.8e19f;      // the latter's square is finite, and after its scale's rounding too

struct AdamTensor {
  void* param;          // states_read / states_write: m in fp32
  const void* grad;     //                             v in fp32
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  uint16_t* copy;
  int64_t n;
  float weight_decay;
  uint32_t flags;
  int32_t chunk0;       // first chunk of this tensor
  int32_t pad;
};

template <int kCap>
struct AdamParams {
  AdamTensor t[kCap];
  int32_t count;
  float beta1, omb1, beta2, omb2, eps;
  const float* hyper;
  int32_t* dev_status;
};

enum class AdamMode { kStep, kRead, kWrite };

// The eight elements of a lane: 4 at base + 4 lane, 4 at base + 128 + 4 lane; elements from `left` on do not exist.
DEV int lane_elem(int i, int lane) { return (i >> 2) * 128 + 4 * lane + (i & 3); }

DEV void load_f32(const float* p, int lane, int left, float (&v)[8]) {
  if (left >= kBlock) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 a = *reinterpret_cast<const float4*>(p + h * 128 + 4 * lane);
      v[4 * h] = a.x; v[4 * h + 1] = a.y; v[4 * h + 2] = a.z; v[4 * h + 3] = a.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = lane_elem(i, lane) < left ? p[lane_elem(i, lane)] : 0.f;
  }
}
DEV void store_f32(float* p, int lane, int left, const float (&v)[8]) {
  if (left >= kBlock) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<float4*>(p + h * 128 + 4 * lane) = make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane_elem(i, lane) < left) p[lane_elem(i, lane)] = v[i];
  }
}
DEV void load_bf16(const uint16_t* p, int lane, int left, float (&v)[8]) {
  if (left >= kBlock) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 a = *reinterpret_cast<const uint2*>(p + h * 128 + 4 * lane);
      v[4 * h] = bf16_bits_to_float(a.x & 0xFFFFu); v[4 * h + 1] = bf16_bits_to_float(a.x >> 16);
      v[4 * h + 2] = bf16_bits_to_float(a.y & 0xFFFFu); v[4 * h + 3] = bf16_bits_to_float(a.y >> 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = lane_elem(i, lane) < left ? bf16_bits_to_float(p[lane_elem(i, lane)]) : 0.f;
  }
}
DEV void store_bf16(uint16_t* p, int lane, int left, const float (&v)[8]) {
  if (left >= kBlock) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<uint2*>(p + h * 128 + 4 * lane) =
          make_uint2(pack_bf16x2(v[4 * h], v[4 * h + 1]), pack_bf16x2(v[4 * h + 2], v[4 * h + 3]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane_elem(i, lane) < left) p[lane_elem(i, lane)] = (uint16_t)(pack_bf16x2(v[i], 0.f) & 0xFFFFu);
  }
}
DEV void load_codes(const uint8_t* p, int lane, int left, uint32_t (&c)[2]) {
  if (left >= kBlock) {
#pragma unroll
    for (int h = 0; h < 2; ++h) c[h] = *reinterpret_cast<const uint32_t*>(p + h * 128 + 4 * lane);
  } else {
    c[0] = c[1] = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane_elem(i, lane) < left) c[i >> 2] |= (uint32_t)p[lane_elem(i, lane)] << (8 * (i & 3));
  }
}
DEV void store_codes(uint8_t* p, int lane, int left, const uint32_t (&c)[2]) {
  if (left >= kBlock) {
#pragma unroll
    for (int h = 0; h < 2; ++h) *reinterpret_cast<uint32_t*>(p + h * 128 + 4 * lane) = c[h];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane_elem(i, lane) < left) p[lane_elem(i, lane)] = (uint8_t)(c[i >> 2] >> (8 * (i & 3)));
  }
}

DEV void decode_m(const uint32_t (&c)[2], float scale, float (&m)[8]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c[q >> 1] >> (16 * (q & 1))), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    parts(pair_of(f.x, f.y) * both(scale), &m[2 * q], &m[2 * q + 1]);
  }
}
// A code's exponent and mantissa bits are those of a half-precision number of twice its value, its exponent counted from 2^-14; 0 is 0.
DEV void decode_v(const uint32_t (&c)[2], float scale, float (&v)[8]) {
  const F2 half_scale = both(0.5f * scale);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint32_t bits = __byte_perm(c[i >> 2], 0u, (i & 2) != 0 ? 0x4342 : 0x4140) * 64u + 0x04000400u;
    const __half2 h = *reinterpret_cast<const __half2*>(&bits), least = __half2(__ushort_as_half(0x0400), __ushort_as_half(0x0400));
    const float2 w = __half22float2(__hmul2(h, __hgt2(h, least)));
    const F2 u = pair_of(w.x, w.y) * half_scale;
    parts(u * u, &v[i], &v[i + 1]);
  }
}

DEV float warp_max(float a) {             // a >= +0: their bits are ordered as they are
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(a)));
}
DEV void encode_m(const float (&m)[8], float f, uint32_t (&c)[2]) {
  c[0] = c[1] = 0u;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float2 x;
    parts(pair_of(m[2 * q], m[2 * q + 1]) * both(f), &x.x, &x.y);
    c[q >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(x, __NV_SATFINITE, __NV_E4M3) << (16 * (q & 1));
  }
}
DEV void encode_v(const float (&u)[8], float f, uint32_t (&c)[2]) {   // u = sqrt(v)
  uint32_t code[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float x[2];
    parts(pair_of(u[i], u[i + 1]) * both(f), &x[0], &x[1]);
#pragma unroll
    for (int k = 0; k < 2; ++k) {          // at most 1.9375 and half a step: code 255; least code of a product above zero: 1
      const uint32_t bits = __float_as_uint(x[k]);
      code[i + k] = (uint32_t)max((int)((bits + 0x3FFFFu + ((bits >> 19) & 1u)) >> 19) - (112 << 4), (int)min(bits, 1u));
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
    c[h] = __byte_perm(__byte_perm(code[4 * h], code[4 * h + 1], 0x0040), __byte_perm(code[4 * h + 2], code[4 * h + 3], 0x0040), 0x5410);
}
// A block's codes and scales from m and u = sqrt(v).  The two scales and the two factors that take values to codes are one division, by a lane each.
// False: a v is infinite.  It is held as the largest whose square is finite: an infinite scale would make NaN of the whole block when it is read.
DEV bool store_states(const AdamTensor& t, int64_t e0, int lane, int left, const float (&m)[8], float (&u)[8]) {
  float am = 0.f, au = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    am = fmaxf(am, fabsf(m[i]));
    au = fmaxf(au, u[i]);
  }
  am = warp_max(am);
  au = warp_max(au);
  const bool fine = au <= kMostFinite;
  if (!fine) {                             // the same in all lanes
    au = kMostRoot;
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = fminf(u[i], kMostRoot);
  }
  const float largest = (lane & 2) != 0 ? au : am, top = (lane & 2) != 0 ? kTopV : kTopM;
  const bool factor = (lane & 1) != 0;
  const float q = largest >= kZeroBlock ? __fdiv_rn(factor ? top : largest, factor ? largest : top) : 0.f;
  uint32_t cm[2], cv[2];
  encode_m(m, __shfl_sync(0xffffffffu, q, 1), cm);
  encode_v(u, __shfl_sync(0xffffffffu, q, 3), cv);
  store_codes(static_cast<uint8_t*>(t.m) + e0, lane, left, cm);
  store_codes(static_cast<uint8_t*>(t.v) + e0, lane, left, cv);
  if (lane == 0) t.m_scale[e0 / kBlock] = q;
  if (lane == 2) t.v_scale[e0 / kBlock] = q;
  return fine;
}

// What a lane reads of a block, as it lies in memory: fetched one block ahead of its use.
struct AdamRaw {
  uint4 g[2], p[2];      // bf16: the first 8 bytes of each
  uint4 m[2], v[2];      // 8 bits: the first 4 bytes of each
  float m_scale, v_scale;
};
template <int kBytes>
DEV void load_raw(const void* base, int64_t e0, int lane, uint4 (&r)[2]) {     // kBytes an element; a whole block
  const char* p = static_cast<const char*>(base) + e0 * kBytes + lane * 4 * kBytes;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (kBytes == 4) r[h] = *reinterpret_cast<const uint4*>(p + h * 512);
    if constexpr (kBytes == 2) { const uint2 a = *reinterpret_cast<const uint2*>(p + h * 256); r[h].x = a.x; r[h].y = a.y; }
    if constexpr (kBytes == 1) r[h].x = *reinterpret_cast<const uint32_t*>(p + h * 128);
  }
}
DEV void raw_f32(const uint4 (&r)[2], float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    v[4 * h] = __uint_as_float(r[h].x); v[4 * h + 1] = __uint_as_float(r[h].y);
    v[4 * h + 2] = __uint_as_float(r[h].z); v[4 * h + 3] = __uint_as_float(r[h].w);
  }
}
DEV void raw_bf16(const uint4 (&r)[2], float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    v[4 * h] = bf16_bits_to_float(r[h].x & 0xFFFFu); v[4 * h + 1] = bf16_bits_to_float(r[h].x >> 16);
    v[4 * h + 2] = bf16_bits_to_float(r[h].y & 0xFFFFu); v[4 * h + 3] = bf16_bits_to_float(r[h].y >> 16);
  }
}

struct AdamStep {
  F2 beta1, omb1, beta2, omb2, decay, clip;
  float eps, step, inv_bias2;
};

// One warp, one block of 256 elements, `left` of which exist; two elements an instruction.  False: a parameter or a v is not finite.
template <bool kEight>
DEV bool adam_block(const AdamTensor& t, const AdamStep& a, int64_t e0, int lane, int left, const float (&g)[8], float (&p)[8], float (&m)[8],
                    float (&v)[8]) {
  float u[8];
  F2 finite = both(0.f);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const F2 gi = pair_of(g[i], g[i + 1]) * a.clip;
    // Products and sums are rounded one by one.  The sums are single ones: packed, they were fused with the products behind them.
    float m0[2], m1[2], v0[2], v1[2];
    parts(pair_of(m[i], m[i + 1]) * a.beta1, &m0[0], &m0[1]);
    parts(gi * a.omb1, &m1[0], &m1[1]);
    parts(pair_of(v[i], v[i + 1]) * a.beta2, &v0[0], &v0[1]);
    parts(gi * a.omb2 * gi, &v1[0], &v1[1]);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      m[i + k] = __fadd_rn(m0[k], m1[k]);
      v[i + k] = __fadd_rn(v0[k], v1[k]);
    }
    u[i] = __fsqrt_rn(v[i]);
    u[i + 1] = __fsqrt_rn(v[i + 1]);
    const F2 by = pair_of(__fdividef(m[i], fmaf(u[i], a.inv_bias2, a.eps)), __fdividef(m[i + 1], fmaf(u[i + 1], a.inv_bias2, a.eps)));
    const F2 pi = fma2(by, both(-a.step), pair_of(p[i], p[i + 1]) * a.decay);
    finite = fma2(pi, both(0.f), finite);        // 0 while every value is finite, NaN otherwise
    if (!kEight) finite = fma2(pair_of(v[i], v[i + 1]), both(0.f), finite);      // g^2 may overflow while m / sqrt(v) does not
    parts(pi, &p[i], &p[i + 1]);
  }
  if (t.flags & MOE_ADAMW_PARAM_BF16) store_bf16(static_cast<uint16_t*>(t.param) + e0, lane, left, p);
  else store_f32(static_cast<float*>(t.param) + e0, lane, left, p);
  if (t.copy != nullptr) store_bf16(t.copy + e0, lane, left, p);
  bool fine = true;
  if constexpr (kEight) {
    fine = store_states(t, e0, lane, left, m, u);
  } else {
    store_f32(static_cast<float*>(t.m) + e0, lane, left, m);
    store_f32(static_cast<float*>(t.v) + e0, lane, left, v);
  }
  return fine && sum_of(finite) == 0.f;
}

// A warp's blocks of a chunk, e0, e0 + step ..  below end.
template <bool kEight>
DEV bool adam_blocks(const AdamTensor& t, const AdamStep& a, int64_t e0, int64_t end, int lane) {
  constexpr int64_t kStride = kAdamThreads / 32 * kBlock;
  const bool g16 = (t.flags & MOE_ADAMW_GRAD_BF16) != 0, p16 = (t.flags & MOE_ADAMW_PARAM_BF16) != 0;
  auto load = [&](int64_t e, AdamRaw& r) {
    if (g16) load_raw<2>(t.grad, e, lane, r.g); else load_raw<4>(t.grad, e, lane, r.g);
    if (p16) load_raw<2>(t.param, e, lane, r.p); else load_raw<4>(t.param, e, lane, r.p);
    load_raw<kEight ? 1 : 4>(t.m, e, lane, r.m);
    load_raw<kEight ? 1 : 4>(t.v, e, lane, r.v);
    if (kEight) { r.m_scale = t.m_scale[e / kBlock]; r.v_scale = t.v_scale[e / kBlock]; }
  };
  float g[8], p[8], m[8], v[8];
  bool fine = true;
  AdamRaw next;
  if (e0 + kBlock <= end) load(e0, next);
  for (; e0 + kBlock <= end; e0 += kStride) {
    if (g16) raw_bf16(next.g, g); else raw_f32(next.g, g);
    if (p16) raw_bf16(next.p, p); else raw_f32(next.p, p);
    if constexpr (kEight) {
      const uint32_t cm[2] = {next.m[0].x, next.m[1].x}, cv[2] = {next.v[0].x, next.v[1].x};
      decode_m(cm, next.m_scale, m);
      decode_v(cv, next.v_scale, v);
    } else {
      raw_f32(next.m, m);
      raw_f32(next.v, v);
    }
    if (e0 + kStride + kBlock <= end) load(e0 + kStride, next);
    fine &= adam_block<kEight>(t, a, e0, lane, kBlock, g, p, m, v);
  }
  if (e0 < end) {                                // the tensor's last elements
    const int left = (int)(end - e0);
    if (g16) load_bf16(static_cast<const uint16_t*>(t.grad) + e0, lane, left, g);
    else load_f32(static_cast<const float*>(t.grad) + e0, lane, left, g);
    if (p16) load_bf16(static_cast<const uint16_t*>(t.param) + e0, lane, left, p);
    else load_f32(static_cast<const float*>(t.param) + e0, lane, left, p);
    if constexpr (kEight) {
      uint32_t cm[2], cv[2];
      load_codes(static_cast<const uint8_t*>(t.m) + e0, lane, left, cm);
      load_codes(static_cast<const uint8_t*>(t.v) + e0, lane, left, cv);
      decode_m(cm, t.m_scale[e0 / kBlock], m);
      decode_v(cv, t.v_scale[e0 / kBlock], v);
    } else {
      load_f32(static_cast<const float*>(t.m) + e0, lane, left, m);
      load_f32(static_cast<const float*>(t.v) + e0, lane, left, v);
    }
    fine &= adam_block<kEight>(t, a, e0, lane, left, g, p, m, v);
  }
  return fine;
}

DEV void read_block(const AdamTensor& t, int64_t e0, int lane) {
  const int left = (int)min(t.n - e0, (int64_t)kBlock);
  uint32_t cm[2], cv[2];
  float m[8], v[8];
  load_codes(static_cast<const uint8_t*>(t.m) + e0, lane, left, cm);
  load_codes(static_cast<const uint8_t*>(t.v) + e0, lane, left, cv);
  decode_m(cm, t.m_scale[e0 / kBlock], m);
  decode_v(cv, t.v_scale[e0 / kBlock], v);
  store_f32(static_cast<float*>(t.param) + e0, lane, left, m);
  store_f32(static_cast<float*>(const_cast<void*>(t.grad)) + e0, lane, left, v);
}

DEV bool write_block(const AdamTensor& t, int64_t e0, int lane) {
  const int left = (int)min(t.n - e0, (int64_t)kBlock);
  float m[8], v[8];
  load_f32(static_cast<const float*>(t.param) + e0, lane, left, m);
  load_f32(static_cast<const float*>(t.grad) + e0, lane, left, v);
  bool fine = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    fine &= fabsf(m[i]) <= kMostFinite && v[i] >= 0.f && v[i] <= kMostFinite;
    v[i] = __fsqrt_rn(v[i]);
  }
  store_states(t, e0, lane, left, m, v);
  return fine;
}

template <AdamMode kMode, int kCap>
__global__ void __launch_bounds__(kAdamThreads, 3)
adamw_kernel(const __grid_constant__ AdamParams<kCap> a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // the tensor of this chunk: the last whose first chunk is not behind it
  const int chunk = (int)blockIdx.x;
  int lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.t[mid].chunk0 <= chunk) lo = mid; else hi = mid;
  }
  const AdamTensor& t = a.t[lo];
  const int64_t first = (int64_t)(chunk - t.chunk0) * kChunk, end = min(first + kChunk, t.n);
  pdl_prologue_done();
  bool fine = true;
  if (kMode == AdamMode::kStep) {
    const float lr = __ldg(a.hyper), bias1 = __ldg(a.hyper + 1), bias2 = __ldg(a.hyper + 2), clip = __ldg(a.hyper + 3);
    const AdamStep s{both(a.beta1), both(a.omb1), both(a.beta2), both(a.omb2), both(__fadd_rn(1.f, -__fmul_rn(lr, t.weight_decay))), both(clip),
                     a.eps, __fdiv_rn(lr, bias1), __fdiv_rn(1.f, __fsqrt_rn(bias2))};
    const int64_t e0 = first + warp * kBlock;
    fine = t.flags & MOE_ADAMW_STATE8 ? adam_blocks<true>(t, s, e0, end, lane) : adam_blocks<false>(t, s, e0, end, lane);
  } else {
    for (int64_t e0 = first + warp * kBlock; e0 < end; e0 += kAdamThreads / 32 * kBlock) {
      if (kMode == AdamMode::kRead) read_block(t, e0, lane);
      else fine &= write_block(t, e0, lane);
    }
  }
  if (kMode != AdamMode::kRead && __any_sync(0xffffffffu, !fine) && lane == 0) set_dev_status(a.dev_status, MOE_ERR_NONFINITE);
}

}  // namespace allocmoe

using namespace allocmoe;

namespace {

constexpr int kMostTensors = 400;        // 80 bytes each
static_assert(sizeof(AdamParams<kMostTensors>) <= 32764, "what a launch's parameters may take");

template <AdamMode kMode, int kCap>
moe_status launch_part(const AdamwArgs& a, int first, int count) {
  AdamParams<kCap> p;
  int64_t chunks = 0;
  for (int k = 0; k < count; ++k) {
    const moe_adamw_tensor& t = a.tensors[first + k];
    AdamTensor& d = p.t[k];
    d.param = t.param;
    d.grad = t.grad;
    if (kMode != AdamMode::kStep) {
      d.param = const_cast<float*>(a.m32[first + k]);
      d.grad = a.v32[first + k];
    }
    d.m = t.m;
    d.v = t.v;
    d.m_scale = t.m_scale;
    d.v_scale = t.v_scale;
    d.copy = t.copy;
    d.n = t.n;
    d.weight_decay = t.weight_decay;
    d.flags = t.flags;
    d.chunk0 = (int32_t)chunks;
    d.pad = 0;
    chunks += (t.n + kChunk - 1) / kChunk;
  }
  p.count = count;
  p.beta1 = (float)a.beta1;
  p.omb1 = (float)(1.0 - a.beta1);
  p.beta2 = (float)a.beta2;
  p.omb2 = (float)(1.0 - a.beta2);
  p.eps = (float)a.eps;
  p.hyper = a.hyper;
  p.dev_status = a.dev_status;
  return launch_dependent(adamw_kernel<kMode, kCap>, dim3((unsigned)chunks), dim3(kAdamThreads), 0, a.stream, 1, p) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}

// The smallest of three parameter blocks that holds the list.
template <AdamMode kMode>
moe_status launch_all(const AdamwArgs& a) {
  for (int first = 0; first < a.count; first += kMostTensors) {
    const int count = a.count - first < kMostTensors ? a.count - first : kMostTensors;
    const moe_status r = count <= 8    ? launch_part<kMode, 8>(a, first, count)
                         : count <= 64 ? launch_part<kMode, 64>(a, first, count)
                                       : launch_part<kMode, kMostTensors>(a, first, count);
    if (r != MOE_OK) return r;
  }
  return MOE_OK;
}

}  // namespace

bool adamw_chunks_ok(const moe_adamw_tensor* tensors, int count) {
  int64_t chunks = 0;
  for (int k = 0; k < count; ++k) {
    if (k % kMostTensors == 0) chunks = 0;
    if (tensors[k].n < 1 || tensors[k].n > ((int64_t)kChunk << 31)) return false;
    chunks += (tensors[k].n + kChunk - 1) / kChunk;
    if (chunks > INT32_MAX) return false;
  }
  return true;
}

moe_status launch_adamw_step(const AdamwArgs& a) { return launch_all<AdamMode::kStep>(a); }
moe_status launch_adamw_read(const AdamwArgs& a) { return launch_all<AdamMode::kRead>(a); }
moe_status launch_adamw_write(const AdamwArgs& a) { return launch_all<AdamMode::kWrite>(a); }
