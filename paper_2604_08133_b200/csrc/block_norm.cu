// The step between two blocks of a residual stack (formulas: allocmoe.h): post-norm, gate, residual scale, residual and the
// next pre-norm in one pass over the rows, forward and backward.
//
// Bound by memory: a forward element moves 8 bytes (10 with a gate for each channel), a backward one 12 (16).  A row is held in
// registers by `tpr` threads, kVec pieces of 8 elements each, so everything is read once; the gains stay in registers over the rows
// that a CTA takes.  Both passes need two dependent sums over the row (y's and then r_out's squares; the three sums behind d_r and
// then the one behind d_y): warps by shuffle, their sums through shared memory, added in warp order by every thread.
//
// Backward, one identity saves a third sum: with q = sum_h sigmoid(gate) w_post y_hat d_r the mean in d_y is scale q / H, the
// row's share of d_scale is q, and a token's gate gets scale (1 - sigmoid) q.
// dw_post, dw_pre and d_scale: every thread adds its columns over the CTA's rows in registers; a second launch adds the CTAs' rows of
// partial sums in order.
//
// Rows come through a ring in shared memory, kStages - 1 of them ahead: a thread copies the 16-byte pieces that it will read itself
// (cp.async), so the ring needs no barrier, only the thread's own wait.  Without it a CTA's loads stood still while it reduced.
#include "common.cuh"
#include "train.h"

namespace allocmoe {

constexpr int kNormMostThreads = 512, kNormMostWarps = kNormMostThreads / 32;
constexpr int kJoinRows = 8;             // threads that share a column in the second launch

DEV void unpack8(const uint4& v, float (&f)[8]) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f[2 * q] = bf16_bits_to_float(u[q] & 0xFFFFu);
    f[2 * q + 1] = bf16_bits_to_float(u[q] >> 16);
  }
}
DEV uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
DEV float sigmoid_of(float g) { return __fdiv_rn(1.f, 1.f + __expf(-g)); }

// kSums sums over the `tpr` threads of a row, which every thread of the CTA takes part in.  Reductions take turns with two buffers:
// a thread that writes one has passed the barrier of the reduction before, behind which nobody reads it any more.
typedef double NormBuf[kNormMostWarps * 2];       // three fp32 sums a warp or one of 64 bits
struct RowSums {
  NormBuf* buf;
  int tpr, turn = 0;
  DEV RowSums(NormBuf* b, int t) : buf(b), tpr(t) {}
  template <typename T, int kSums>
  DEV void operator()(T (&s)[kSums]) { sum(s, reinterpret_cast<T*>(buf[turn ^= 1]), tpr); }
  template <typename T, int kSums>
  static DEV void sum(T (&s)[kSums], T* buf, int tpr);
};
template <typename T, int kSums>
DEV void RowSums::sum(T (&s)[kSums], T* buf, int tpr) {
#pragma unroll
  for (int i = 0; i < kSums; ++i)
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) s[i] += __shfl_xor_sync(0xffffffffu, s[i], d);
  if (tpr == 32) return;
  const int warp = threadIdx.x >> 5, per_row = tpr >> 5, w0 = warp / per_row * per_row;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < kSums; ++i) buf[warp * kSums + i] = s[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSums; ++i) s[i] = (T)0;
  for (int w = 0; w < per_row; ++w)
#pragma unroll
    for (int i = 0; i < kSums; ++i) s[i] += buf[(w0 + w) * kSums + i];
}

struct NormParams {
  const uint4* r;
  const uint4* y;
  const float4* w_post;
  const uint16_t* gate;
  const float* scale;
  const float4* w_pre;
  uint4* r_out;
  uint4* n_out;
  const uint4* d_n;
  const uint4* d_r_out;
  uint4* d_r;
  uint4* d_y;
  uint16_t* d_gate;
  float* partial;       // [CTAs][2H + 8]: dw_post, dw_pre, d_scale (64 bits) of the CTA's rows; nullptr: not wanted
  int T, H, gate_cols, tpr, rows;
  float eps;
  bool normalise_y;
};

// The thread's ring: kArrays arrays of kVec pieces a stage.  Piece k of a row is 16-byte vector c0 + k * tpr.
template <int kVec, int kArrays, int kStages>
struct NormRing {
  uint4* mine;           // of stage 0, array 0, piece 0; the CTA's threads lie next to each other
  int threads;
  DEV NormRing(void* smem) : mine(static_cast<uint4*>(smem) + threadIdx.x), threads(blockDim.x) {}
  DEV uint4* at(int stage, int array, int k) const { return mine + (size_t)((stage * kArrays + array) * kVec + k) * threads; }
  // arrays that are nullptr are left out; rows and pieces that do not exist are not copied
  DEV void fetch(int stage, const uint4* const (&src)[kArrays], size_t row_at, bool row_ok, int c0, int tpr, int nv) const {
#pragma unroll
    for (int a = 0; a < kArrays; ++a)
#pragma unroll
      for (int k = 0; k < kVec; ++k)
        if (row_ok && src[a] != nullptr && c0 + k * tpr < nv) cp_async_16(at(stage, a, k), src[a] + row_at + c0 + k * tpr, true);
    cp_async_commit();
  }
  DEV uint4 get(int stage, int array, int k, bool exists) const { return exists ? *at(stage, array, k) : make_uint4(0, 0, 0, 0); }
};
// S - 1 rows ahead while two CTAs of 512 threads (forward: 3 arrays) fit an SM; at two pieces a thread the backward pass has room for two stages.
template <int kVec, int kArrays>
constexpr int kNormStages = kVec * kArrays <= 6 ? 4 : 2;

DEV void load_gain(const float4* w, int v, float (&f)[8]) {
  if (w == nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 1.f;
    return;
  }
  const float4 a = __ldg(w + 2 * v), b = __ldg(w + 2 * v + 1);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

template <int kVec>
__global__ void __launch_bounds__(kNormMostThreads)
block_norm_kernel(const NormParams p) {
  extern __shared__ __align__(16) unsigned char smem_dyn[];
  __shared__ NormBuf buf[2];
  RowSums row_sums(buf, p.tpr);
  const int row_in = threadIdx.x / p.tpr, c0 = threadIdx.x % p.tpr, nv = p.H / 8;
  const float inv_h = 1.f / (float)p.H;
  pdl_prologue_done();
  float w_post[kVec][8], w_pre[kVec][8];
#pragma unroll
  for (int k = 0; k < kVec; ++k)
    if (c0 + k * p.tpr < nv) {
      if (p.y != nullptr) load_gain(p.w_post, c0 + k * p.tpr, w_post[k]);
      if (p.n_out != nullptr) load_gain(p.w_pre, c0 + k * p.tpr, w_pre[k]);
    }
  const float scale = p.y != nullptr && p.scale != nullptr ? __ldg(p.scale) : 1.f;
  constexpr int kStages = kNormStages<kVec, 3>;
  const NormRing<kVec, 3, kStages> ring(smem_dyn);
  const bool wide_gate = p.y != nullptr && p.gate_cols > 1;
  const uint4* const src[3] = {p.r, p.y, wide_gate ? reinterpret_cast<const uint4*>(p.gate) : nullptr};
  const long long step = (long long)gridDim.x * p.rows, first = (long long)blockIdx.x * p.rows;
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s)
    ring.fetch(s, src, (size_t)(first + s * step + row_in) * nv, first + s * step + row_in < p.T, c0, p.tpr, nv);
  int stage = 0;
  float gate_next = 0.f;
  if (p.y != nullptr && p.gate_cols == 1 && first + row_in < p.T) gate_next = bf16_bits_to_float(p.gate[first + row_in]);
  for (long long base = first; base < p.T; base += step) {
    const long long row = base + row_in, ahead = row + (kStages - 1) * step;
    const bool mine = row < p.T;
    const size_t at = (size_t)row * nv;
    uint4 r[kVec], y[kVec], g[kVec];
    const float one_gate = p.gate_cols == 1 ? sigmoid_of(gate_next) : 1.f;
    if (p.y != nullptr && p.gate_cols == 1 && row + step < p.T) gate_next = bf16_bits_to_float(p.gate[row + step]);
    ring.fetch((stage + kStages - 1) % kStages, src, (size_t)ahead * nv, ahead < p.T, c0, p.tpr, nv);
    cp_async_wait<kStages - 1>();
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const bool has = mine && c0 + k * p.tpr < nv;
      r[k] = ring.get(stage, 0, k, has);
      y[k] = ring.get(stage, 1, k, has && p.y != nullptr);
      g[k] = ring.get(stage, 2, k, has && wide_gate);
    }
    stage = (stage + 1) % kStages;
    float ss[1] = {0.f};
    if (p.y != nullptr) {
      float inv_y = 1.f;
      if (p.normalise_y) {
        float sy[1] = {0.f};
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
          float f[8];
          unpack8(y[k], f);
#pragma unroll
          for (int e = 0; e < 8; ++e) sy[0] = fmaf(f[e], f[e], sy[0]);
        }
        row_sums(sy);
        inv_y = __frsqrt_rn(fmaf(sy[0], inv_h, p.eps));
      }
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        const int v = c0 + k * p.tpr;
        if (v >= nv) continue;
        float fr[8], fy[8], fg[8];
        unpack8(r[k], fr);
        unpack8(y[k], fy);
        unpack8(g[k], fg);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float sg = p.gate_cols > 1 ? sigmoid_of(fg[e]) : p.gate_cols == 1 ? one_gate : 1.f;
          fr[e] = fmaf(scale * sg, fy[e] * inv_y * w_post[k][e], fr[e]);
        }
        r[k] = pack8(fr);
        if (mine) p.r_out[at + v] = r[k];
      }
    }
    if (p.n_out == nullptr) continue;
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      float f[8];
      unpack8(r[k], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss[0] = fmaf(f[e], f[e], ss[0]);
    }
    row_sums(ss);
    const float inv_r = __frsqrt_rn(fmaf(ss[0], inv_h, p.eps));
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const int v = c0 + k * p.tpr;
      if (!mine || v >= nv) continue;
      float f[8];
      unpack8(r[k], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= inv_r * w_pre[k][e];
      p.n_out[at + v] = pack8(f);
    }
  }
}

template <int kVec>
__global__ void __launch_bounds__(kNormMostThreads)
block_norm_backward_kernel(const NormParams p) {
  __shared__ NormBuf buf[2];
  RowSums row_sums(buf, p.tpr);
  extern __shared__ __align__(16) unsigned char smem_dyn[];
  float* joined = reinterpret_cast<float*>(smem_dyn);   // behind the rows: [rows][2H + 8], where a CTA takes several rows at a time
  const int row_in = threadIdx.x / p.tpr, c0 = threadIdx.x % p.tpr, nv = p.H / 8;
  const float inv_h = 1.f / (float)p.H;
  pdl_prologue_done();
  float w_post[kVec][8], w_pre[kVec][8], sum_post[kVec][8], sum_pre[kVec][8];
  double sum_scale = 0.0;
#pragma unroll
  for (int k = 0; k < kVec; ++k) {
    if (c0 + k * p.tpr < nv) {
      if (p.y != nullptr) load_gain(p.w_post, c0 + k * p.tpr, w_post[k]);
      if (p.d_n != nullptr) load_gain(p.w_pre, c0 + k * p.tpr, w_pre[k]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum_post[k][e] = sum_pre[k][e] = 0.f;
  }
  const float scale = p.y != nullptr && p.scale != nullptr ? __ldg(p.scale) : 1.f;
  constexpr int kStages = kNormStages<kVec, 5>;
  const NormRing<kVec, 5, kStages> ring(smem_dyn);
  const bool wide_gate = p.y != nullptr && p.gate_cols > 1;
  const uint4* const src[5] = {p.d_n != nullptr ? p.r : nullptr, p.d_n, p.d_r_out, p.y, wide_gate ? reinterpret_cast<const uint4*>(p.gate) : nullptr};
  const long long step = (long long)gridDim.x * p.rows, first = (long long)blockIdx.x * p.rows;
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s)
    ring.fetch(s, src, (size_t)(first + s * step + row_in) * nv, first + s * step + row_in < p.T, c0, p.tpr, nv);
  int stage = 0;
  float gate_next = 0.f;
  if (p.y != nullptr && p.gate_cols == 1 && first + row_in < p.T) gate_next = bf16_bits_to_float(p.gate[first + row_in]);
  for (long long base = first; base < p.T; base += step) {
    const long long row = base + row_in, ahead = row + (kStages - 1) * step;
    const bool mine = row < p.T;
    const size_t at = (size_t)row * nv;
    uint4 r[kVec], y[kVec], g[kVec], dn[kVec], dr[kVec];
    const float one_gate = p.gate_cols == 1 ? sigmoid_of(gate_next) : 1.f;
    if (p.y != nullptr && p.gate_cols == 1 && row + step < p.T) gate_next = bf16_bits_to_float(p.gate[row + step]);
    ring.fetch((stage + kStages - 1) % kStages, src, (size_t)ahead * nv, ahead < p.T, c0, p.tpr, nv);
    cp_async_wait<kStages - 1>();
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const bool has = mine && c0 + k * p.tpr < nv;
      r[k] = ring.get(stage, 0, k, has && p.d_n != nullptr);
      dn[k] = ring.get(stage, 1, k, has && p.d_n != nullptr);
      dr[k] = ring.get(stage, 2, k, has && p.d_r_out != nullptr);
      y[k] = ring.get(stage, 3, k, has && p.y != nullptr);
      g[k] = ring.get(stage, 4, k, has && wide_gate);
    }
    stage = (stage + 1) % kStages;
    // sums of r^2, a r and y^2
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      if (c0 + k * p.tpr >= nv) continue;
      float fr[8], fn[8], fy[8];
      unpack8(r[k], fr);
      unpack8(dn[k], fn);
      unpack8(y[k], fy);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[0] = fmaf(fr[e], fr[e], s[0]);
        if (p.d_n != nullptr) s[1] = fmaf(fn[e] * w_pre[k][e], fr[e], s[1]);
        s[2] = fmaf(fy[e], fy[e], s[2]);
      }
    }
    row_sums(s);
    const float inv_r = __frsqrt_rn(fmaf(s[0], inv_h, p.eps)), inv_y = p.normalise_y ? __frsqrt_rn(fmaf(s[2], inv_h, p.eps)) : 1.f;
    const float mean = inv_r * inv_r * inv_r * (s[1] * inv_h);       // mean_h(a r_hat) / rms^2, taken times r below
    float f_dr[kVec][8];
    double q[1] = {0.0};      // d_scale is a sum over the whole batch in which most cancels: 64 bits beyond a thread's own terms
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const int v = c0 + k * p.tpr;
      if (v >= nv) continue;
      float fr[8], fn[8], fy[8], fg[8];
      unpack8(dr[k], f_dr[k]);
      if (p.d_n != nullptr) {
        unpack8(r[k], fr);
        unpack8(dn[k], fn);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f_dr[k][e] += inv_r * (fn[e] * w_pre[k][e]) - mean * fr[e];
          sum_pre[k][e] = fmaf(fn[e], fr[e] * inv_r, sum_pre[k][e]);
        }
      }
      if (mine && p.d_r != nullptr) p.d_r[at + v] = pack8(f_dr[k]);
      if (p.y != nullptr) {
        unpack8(y[k], fy);
        unpack8(g[k], fg);
        float part[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float sg = p.gate_cols > 1 ? sigmoid_of(fg[e]) : p.gate_cols == 1 ? one_gate : 1.f;
          const float t = sg * f_dr[k][e] * (fy[e] * inv_y);
          sum_post[k][e] = fmaf(scale, t, sum_post[k][e]);
          part[e] = t * w_post[k][e];
        }
        q[0] += (double)(((part[0] + part[1]) + (part[2] + part[3])) + ((part[4] + part[5]) + (part[6] + part[7])));
      }
    }
    if (p.y == nullptr) continue;
    row_sums(q);
    if (c0 == 0 && mine) {
      sum_scale += q[0];
      if (p.gate_cols == 1 && p.d_gate != nullptr) p.d_gate[row] = (uint16_t)(pack_bf16x2(scale * (1.f - one_gate) * (float)q[0], 0.f) & 0xFFFFu);
    }
    const float mean_y = p.normalise_y ? scale * (float)q[0] * inv_h : 0.f;
    if (p.d_y == nullptr && (p.d_gate == nullptr || p.gate_cols <= 1)) continue;
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const int v = c0 + k * p.tpr;
      if (!mine || v >= nv) continue;
      float fy[8], fg[8], dy[8], dg[8];
      unpack8(y[k], fy);
      unpack8(g[k], fg);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float sg = p.gate_cols > 1 ? sigmoid_of(fg[e]) : p.gate_cols == 1 ? one_gate : 1.f;
        const float y_hat = fy[e] * inv_y, b = scale * w_post[k][e] * f_dr[k][e];
        dy[e] = inv_y * (b * sg - y_hat * mean_y);
        dg[e] = b * y_hat * (sg * (1.f - sg));
      }
      if (p.d_y != nullptr) p.d_y[at + v] = pack8(dy);
      if (p.d_gate != nullptr && p.gate_cols > 1) reinterpret_cast<uint4*>(p.d_gate)[at + v] = pack8(dg);
    }
  }
  if (p.partial == nullptr) return;
  // the CTA's sums: its row groups one after the other
  const size_t width = 2 * (size_t)p.H + 8;
  float* out = p.partial + (size_t)blockIdx.x * width;
  if (p.rows > 1) {
    cp_async_wait<0>();
    __syncthreads();                     // the ring's place is free
    float* own = joined + row_in * width;
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const int v = c0 + k * p.tpr;
      if (v >= nv) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) { own[v * 8 + e] = sum_post[k][e]; own[p.H + v * 8 + e] = sum_pre[k][e]; }
    }
    if (c0 == 0) *reinterpret_cast<double*>(own + 2 * p.H) = sum_scale;
    __syncthreads();
    if (threadIdx.x == 0) {
      double a = 0.0;
      for (int w = 0; w < p.rows; ++w) a += *reinterpret_cast<const double*>(joined + w * width + 2 * p.H);
      *reinterpret_cast<double*>(out + 2 * p.H) = a;
    }
    for (int c = threadIdx.x; c < 2 * p.H; c += blockDim.x) {
      float a = 0.f;
      for (int w = 0; w < p.rows; ++w) a += joined[w * width + c];
      out[c] = a;
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < kVec; ++k) {
    const int v = c0 + k * p.tpr;
    if (v >= nv) continue;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      reinterpret_cast<float4*>(out)[2 * v + h] = make_float4(sum_post[k][4 * h], sum_post[k][4 * h + 1], sum_post[k][4 * h + 2], sum_post[k][4 * h + 3]);
      reinterpret_cast<float4*>(out + p.H)[2 * v + h] = make_float4(sum_pre[k][4 * h], sum_pre[k][4 * h + 1], sum_pre[k][4 * h + 2], sum_pre[k][4 * h + 3]);
    }
  }
  if (c0 == 0) *reinterpret_cast<double*>(out + 2 * p.H) = sum_scale;
}

// Columns of the CTAs' partial sums: 32 columns a CTA, kJoinRows threads a column, their sums joined in order.
__global__ void __launch_bounds__(32 * kJoinRows)
block_norm_join_kernel(const float* __restrict__ partial, int n, int H, float* dw_post, float* dw_pre, float* d_scale) {
  __shared__ double part[kJoinRows][33];
  const int c = blockIdx.x * 32 + threadIdx.x, g = threadIdx.y;
  const size_t width = 2 * (size_t)H + 8;
  pdl_prologue_done();
  double a = 0.0;
  if (c < 2 * H)
    for (int i = g; i < n; i += kJoinRows) a += (double)partial[(size_t)i * width + c];
  else if (c == 2 * H)
    for (int i = g; i < n; i += kJoinRows) a += *reinterpret_cast<const double*>(partial + (size_t)i * width + c);
  part[g][threadIdx.x] = a;
  __syncthreads();
  if (g != 0 || c > 2 * H) return;
  a = 0.0;
#pragma unroll
  for (int i = 0; i < kJoinRows; ++i) a += part[i][threadIdx.x];
  if (c < H) { if (dw_post != nullptr) dw_post[c] = (float)a; }
  else if (c < 2 * H) { if (dw_pre != nullptr) dw_pre[c - H] = (float)a; }
  else if (d_scale != nullptr) d_scale[0] = (float)a;
}

}  // namespace allocmoe

using namespace allocmoe;

namespace {

constexpr size_t kMostNormSmem = 200 * 1024;      // 4 stages x 3 arrays x 2 pieces x 512 threads x 16 bytes: 192 KB

struct NormPlan { int vec, tpr, rows; unsigned grid; size_t smem; };

// One piece of 8 elements a thread up to H 4096 (512 threads a row), two beyond (H 8192).  Rows below 128 threads share a CTA.  As many CTAs
// as are resident: of 512 threads two an SM forward (64 registers), one backward; of 1024 threads' worth of smaller ones likewise.
NormPlan plan_of(const moe_norm_shape* s, bool backward) {
  NormPlan n{};
  const int nv = s->H / 8;
  n.vec = nv > 512 ? 2 : 1;
  n.tpr = ((nv + n.vec - 1) / n.vec + 31) / 32 * 32;
  n.rows = n.tpr >= 128 ? 1 : 128 / n.tpr;
  if (n.rows > s->T) n.rows = s->T;
  const int threads = n.tpr * n.rows, most = (backward ? 640 : 1024) / n.vec;     // threads an SM holds, by registers
  const long long ctas = ((long long)s->T + n.rows - 1) / n.rows, resident = 148ll * (most / threads > 0 ? most / threads : 1);
  n.grid = (unsigned)(ctas < resident ? ctas : resident);
  const int arrays = backward ? 5 : 3, stages = n.vec * arrays <= 6 ? 4 : 2;
  n.smem = (size_t)stages * arrays * n.vec * threads * 16;
  const size_t join = backward && n.rows > 1 ? n.rows * (2 * (size_t)s->H + 8) * sizeof(float) : 0;    // rows * H <= 1024: under 9 KB
  if (n.smem < join) n.smem = join;
  return n;
}

NormParams params_of(const BlockNormArgs& a, const NormPlan& n) {
  NormParams p{};
  const moe_norm_shape* s = a.s;
  p.r = reinterpret_cast<const uint4*>(a.r);
  p.y = reinterpret_cast<const uint4*>(a.y);
  p.w_post = reinterpret_cast<const float4*>(a.w_post);
  p.gate = a.gate;
  p.scale = a.scale;
  p.w_pre = reinterpret_cast<const float4*>(a.w_pre);
  p.r_out = reinterpret_cast<uint4*>(a.r_out);
  p.n_out = reinterpret_cast<uint4*>(a.n_out);
  p.d_n = reinterpret_cast<const uint4*>(a.d_n);
  p.d_r_out = reinterpret_cast<const uint4*>(a.d_r_out);
  p.d_r = reinterpret_cast<uint4*>(a.d_r);
  p.d_y = reinterpret_cast<uint4*>(a.d_y);
  p.d_gate = a.d_gate;
  p.T = s->T;
  p.H = s->H;
  p.gate_cols = a.gate != nullptr ? s->gate_cols : 0;
  p.tpr = n.tpr;
  p.rows = n.rows;
  p.eps = s->eps;
  p.normalise_y = (s->flags & MOE_NORM_Y_AS_IS) == 0;
  return p;
}

}  // namespace

size_t block_norm_workspace_bytes(const moe_norm_shape* s) {
  return (size_t)plan_of(s, true).grid * (2 * (size_t)s->H + 8) * sizeof(float);
}

moe_status launch_block_norm(const BlockNormArgs& a) {
  const NormPlan n = plan_of(a.s, false);
  const NormParams p = params_of(a, n);
  static PerDeviceOnce once1, once2;
  auto kernel = n.vec == 1 ? block_norm_kernel<1> : block_norm_kernel<2>;
  if (!ensure_dynamic_smem(kernel, kMostNormSmem, n.vec == 1 ? once1 : once2)) return MOE_ERR_CUDA;
  return launch_dependent(kernel, dim3(n.grid), dim3((unsigned)(n.tpr * n.rows)), n.smem, a.stream, 1, p) == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

moe_status launch_block_norm_backward(const BlockNormArgs& a) {
  const NormPlan n = plan_of(a.s, true);
  NormParams p = params_of(a, n);
  const bool sums = a.dw_post != nullptr || a.dw_pre != nullptr || a.d_scale != nullptr;
  p.partial = sums ? static_cast<float*>(a.ws) : nullptr;
  static PerDeviceOnce once1, once2;
  auto kernel = n.vec == 1 ? block_norm_backward_kernel<1> : block_norm_backward_kernel<2>;
  if (!ensure_dynamic_smem(kernel, kMostNormSmem, n.vec == 1 ? once1 : once2)) return MOE_ERR_CUDA;
  if (launch_dependent(kernel, dim3(n.grid), dim3((unsigned)(n.tpr * n.rows)), n.smem, a.stream, 1, p) != cudaSuccess) return MOE_ERR_CUDA;
  if (!sums) return MOE_OK;
  return launch_dependent(block_norm_join_kernel, dim3((unsigned)((2 * a.s->H + 1 + 31) / 32)), dim3(32, kJoinRows), 0, a.stream, 1,
                          static_cast<const float*>(p.partial), (int)n.grid, (int)a.s->H, a.dw_post, a.dw_pre, a.d_scale) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}
