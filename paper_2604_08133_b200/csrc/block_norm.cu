// The step between two blocks of a residual stack (formulas: allocmoe.h): post-norm, gate, residual scale, residual and the
// next pre-norm in one pass over the rows, forward and backward.
//
// A forward element moves 8 bytes (10 with a gate for each channel), a backward one 12 (16); each is read once.  A row belongs to `tpr`
// threads, one or two pieces of 8 elements each, with the gains in registers over the rows that a CTA takes.  Both passes need two
// dependent sums over the row (y's and then r_out's squares; the three sums behind d_r and then the one behind d_y): warps by shuffle,
// their sums through shared memory, added in warp order by every thread.
//
// What bounds it after memory is the number of instructions: two elements an instruction (fma.rn.f32x2) and two pieces a thread, which halves
// the reductions' share.  8192 rows of 4096 with a gate for each channel: 108 us with one element an instruction and an IEEE division in
// the sigmoid, 96 with an approximate one, 72 with two pieces a thread, 56 with two elements an instruction and a barrier a row: 6.0 TB/s.
// Backward, 4099 rows of 2048 and one gate each: 26.2 us, 16 384 of them 78 (5.2 TB/s).  One CTA of 512 threads an SM; the pieces are read
// from the ring at each use and arrays that the call has not are zeros there (kept in registers they spilled at 128 a thread: 4099 rows of 4096 80 us,
// 57 read again, 50 without the selects, 47 with 32-bit row numbers and a ring whose places are constants).  Copies of whole rows by the bulk engine,
// two to four rows ahead, took as long: it waits for instructions (0.5 a scheduler and clock), not for memory.
//
// Backward, one identity saves a third sum: with q = sum_h sigmoid(gate) w_post y_hat d_r the mean in d_y is scale q / H, the
// row's share of d_scale is q, and a token's gate gets scale (1 - sigmoid) q.
// dw_post, dw_pre and d_scale: every thread adds its columns over its rows in registers, the CTA its threads of a column in shared memory; a
// second launch adds the CTAs' rows of partial sums in order.
//
// Rows come through a ring in shared memory, kStages - 1 of them ahead: a thread copies the 16-byte pieces that it will read itself
// (cp.async), so the ring needs no barrier, only the thread's own wait.
#include "common.cuh"
#include "train.h"

namespace allocmoe {

constexpr int kNormMostThreads = 512, kNormMostWarps = kNormMostThreads / 32;
constexpr int kJoinRows = 32;            // threads that share a column in the second launch (16: 27.2 us for 26.6 in all, 8: 29.6)
static_assert(5 * kJoinRows >= 148, "a row of partial sums for each CTA");

// Eight bf16 of a piece as four pairs, and back.
DEV void unpack(const uint4& v, F2 (&f)[4]) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = pair_of(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xFFFF0000u));
}
DEV uint4 pack(const F2 (&f)[4]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    parts(f[i], &lo, &hi);
    u[i] = pack_bf16x2(lo, hi);
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}
DEV float sigmoid_of(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }
// The sigmoid and one minus it, from one exponential: the difference itself cancels from a gate of 8 on and is zero from 17 on.  A shut gate's infinite
// exponential times its sigmoid of zero is NaN, which the minimum turns into one.
DEV float sigmoid_of(float g, float* rest) {
  const float e = __expf(-g), sg = __fdividef(1.f, 1.f + e);
  *rest = fminf(e * sg, 1.f);
  return sg;
}
DEV F2 sigmoid_of(const F2& g) {
  float lo, hi;
  parts(g, &lo, &hi);
  return pair_of(sigmoid_of(lo), sigmoid_of(hi));
}

// Sums over the `tpr` threads of a row, which all of them call: warps by shuffle, the warps' sums through shared memory, kSums rows of 16.
// Rows that share a CTA each have a barrier of their own.  Reductions take turns with two buffers: a thread that writes one has passed
// the barrier of the reduction before, behind which nobody reads it any more.
typedef double NormBuf[kNormMostWarps * 5 / 2];   // three fp32 sums a warp and one of 64 bits
struct RowSums {
  unsigned char* mine;   // of this row: two buffers
  int tpr, warp, warps, barrier, turn = 0;
  DEV RowSums(NormBuf (*buf)[2], int t) : tpr(t) {
    const int row_in = threadIdx.x / t;
    mine = reinterpret_cast<unsigned char*>(buf[row_in]);
    warps = t >> 5;
    warp = (threadIdx.x >> 5) - row_in * warps;
    barrier = 1 + row_in;
    // sums of warps that a row does not have stay zero
    for (int i = threadIdx.x - row_in * t; i < 2 * kNormMostWarps * 5 / 2; i += t) reinterpret_cast<double*>(mine)[i] = 0.0;
    sync();
  }
  DEV void sync() const { asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(tpr) : "memory"); }
  template <int kSums>
  DEV void operator()(float (&s)[kSums]) {
#pragma unroll
    for (int i = 0; i < kSums; ++i)
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) s[i] += __shfl_xor_sync(0xffffffffu, s[i], d);
    if (tpr == 32) return;
    float* b = reinterpret_cast<float*>(mine + (turn ^= 1) * sizeof(NormBuf));
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int i = 0; i < kSums; ++i) b[i * kNormMostWarps + warp] = s[i];
    sync();
#pragma unroll
    for (int i = 0; i < kSums; ++i) s[i] = 0.f;
#pragma unroll 1
    for (int w = 0; w < warps; w += 4)
#pragma unroll
      for (int i = 0; i < kSums; ++i) {
        const float4 v = *reinterpret_cast<const float4*>(b + i * kNormMostWarps + w);
        s[i] += (v.x + v.y) + (v.z + v.w);
      }
  }
  DEV double operator()(double s) {      // its buffers lie behind those of the fp32 sums: nothing else is ever written there
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if (tpr == 32) return s;
    double* b = reinterpret_cast<double*>(mine + turn * sizeof(NormBuf)) + kNormMostWarps * 3 / 2;
    if ((threadIdx.x & 31) == 0) b[warp] = s;
    sync();
    s = 0.0;
#pragma unroll 1
    for (int w = 0; w < warps; w += 2) {
      const double2 v = *reinterpret_cast<const double2*>(b + w);
      s += v.x + v.y;
    }
    return s;
  }
};

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

// The thread's ring: kArrays arrays of kVec pieces a stage.  Piece k of a row is 16-byte vector c0 + k * tpr; kFull: every piece exists.
template <int kVec, int kMax, int kArrays, int kStages, bool kFull>
struct NormRing {
  uint4* mine;           // of stage 0, array 0, piece 0; the CTA's threads lie next to each other
  int tpr, has;                      // has: pieces of this thread that exist
  size_t next, step;                 // the thread's first piece of the next row to fetch, the same in all arrays; from row to row
  DEV NormRing(void* smem, const NormParams& p, long long row, int c0)
      : mine(static_cast<uint4*>(smem) + threadIdx.x), tpr(p.tpr) {
    const int nv = p.H / 8;
    has = kFull ? kVec : c0 >= nv ? 0 : min(kVec, (nv - 1 - c0) / tpr + 1);
    step = (size_t)gridDim.x * p.rows * nv;
    next = (size_t)row * nv + c0;
  }
  DEV bool piece(int k) const { return kFull || k < has; }
  DEV uint4* at(int stage, int array, int k) const { return mine + ((stage * kArrays + array) * kVec + k) * kMax; }
  // arrays that are nullptr are left out
  DEV void fetch(int stage, bool row_ok, const void* const (&arrays)[kArrays]) {
    if (row_ok) {
#pragma unroll
      for (int a = 0; a < kArrays; ++a)
        if (arrays[a] != nullptr) {
#pragma unroll
          for (int k = 0; k < kVec; ++k)
            if (piece(k)) cp_async_16(at(stage, a, k), static_cast<const uint4*>(arrays[a]) + next + k * tpr, true);
        }
    }
    next += step;
    cp_async_commit();
  }
  // arrays that are left out read as zeros
  DEV void clear(const void* const (&arrays)[kArrays]) const {
    for (int s = 0; s < kStages; ++s)
      for (int a = 0; a < kArrays; ++a)
        if (arrays[a] == nullptr)
          for (int k = 0; k < kVec; ++k) *at(s, a, k) = make_uint4(0, 0, 0, 0);
  }
  DEV uint4 get(int stage, int array, int k, bool present = true) const { return present && piece(k) ? *at(stage, array, k) : make_uint4(0, 0, 0, 0); }
};
// Stages of the rings: one row ahead.  More did not pay: backward 34.2 us with three, 31.3 with two; forward 57.8 with four, 56.3 with two.
constexpr int kForwardStages = 2, kBackwardStages = 2;
constexpr int kBackwardRows = 15;        // rows that a CTA of the backward pass takes at a time, at most: a named barrier each

DEV void load_gain(const float4* w, int v, F2 (&f)[4]) {
  if (w == nullptr) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = both(1.f);
    return;
  }
  const float4 a = __ldg(w + 2 * v), b = __ldg(w + 2 * v + 1);
  f[0] = pair_of(a.x, a.y);
  f[1] = pair_of(a.z, a.w);
  f[2] = pair_of(b.x, b.y);
  f[3] = pair_of(b.z, b.w);
}

// kMax: threads a CTA may have; narrow rows get more registers a thread.
template <int kVec, int kMax, bool kFull>
__global__ void __launch_bounds__(kMax, kMax <= 128 ? 4 : 1)
block_norm_kernel(const NormParams p) {
  extern __shared__ __align__(16) unsigned char smem_dyn[];
  __shared__ __align__(16) NormBuf buf[4][2];    // at most four rows share a CTA
  RowSums row_sums(buf, p.tpr);
  const int row_in = threadIdx.x / p.tpr, c0 = threadIdx.x % p.tpr, nv = p.H / 8;
  const float inv_h = 1.f / (float)p.H;
  pdl_prologue_done();
  F2 w_post[kVec][4], w_pre[kVec][4];
#pragma unroll
  for (int k = 0; k < kVec; ++k)
    if (c0 + k * p.tpr < nv) {
      if (p.y != nullptr) load_gain(p.w_post, c0 + k * p.tpr, w_post[k]);
      if (p.n_out != nullptr) load_gain(p.w_pre, c0 + k * p.tpr, w_pre[k]);
    }
  const float scale = p.y != nullptr && p.scale != nullptr ? __ldg(p.scale) : 1.f;
  constexpr int kStages = kForwardStages;
  const bool has_y = p.y != nullptr, one_gate = has_y && p.gate_cols == 1, wide_gate = has_y && p.gate_cols > 1;
  const long long step = (long long)gridDim.x * p.rows;
  long long row = (long long)blockIdx.x * p.rows + row_in;
  const void* const arrays[3] = {p.r, p.y, wide_gate ? p.gate : nullptr};
  NormRing<kVec, kMax, 3, kStages, kFull> ring(smem_dyn, p, row, c0);
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) ring.fetch(s, row + s * step < p.T, arrays);
  int stage = 0;
  float gate_next = one_gate && row < p.T ? bf16_bits_to_float(p.gate[row]) : 0.f;
  for (; row < p.T; row += step) {
    const size_t at = (size_t)row * nv + c0;
    const float factor = one_gate ? scale * sigmoid_of(gate_next) : scale;
    if (one_gate && row + step < p.T) gate_next = bf16_bits_to_float(p.gate[row + step]);
    ring.fetch(stage == 0 ? kStages - 1 : stage - 1, row + (kStages - 1) * step < p.T, arrays);
    cp_async_wait<kStages - 1>();
    uint4 r[kVec], y[kVec];
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      r[k] = ring.get(stage, 0, k);
      y[k] = ring.get(stage, 1, k, has_y);
    }
    if (has_y) {
      float inv_y = 1.f;
      if (p.normalise_y) {
        F2 s2 = both(0.f);
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
          F2 f[4];
          unpack(y[k], f);
#pragma unroll
          for (int e = 0; e < 4; ++e) s2 = fma2(f[e], f[e], s2);
        }
        float s[1] = {sum_of(s2)};
        row_sums(s);
        inv_y = rsqrtf(fmaf(s[0], inv_h, p.eps));
      }
      const F2 c = both(factor * inv_y);
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        if (!ring.piece(k)) continue;
        F2 fr[4], fy[4];
        unpack(r[k], fr);
        unpack(y[k], fy);
        if (wide_gate) {
          F2 g[4];
          unpack(ring.get(stage, 2, k), g);
#pragma unroll
          for (int e = 0; e < 4; ++e) fy[e] = fy[e] * sigmoid_of(g[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) fr[e] = fma2(fy[e] * w_post[k][e], c, fr[e]);
        r[k] = pack(fr);
        p.r_out[at + k * p.tpr] = r[k];
      }
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (p.n_out == nullptr) continue;
    F2 s2 = both(0.f);
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      F2 f[4];
      unpack(r[k], f);
#pragma unroll
      for (int e = 0; e < 4; ++e) s2 = fma2(f[e], f[e], s2);
    }
    float s[1] = {sum_of(s2)};
    row_sums(s);
    const F2 inv_r = both(rsqrtf(fmaf(s[0], inv_h, p.eps)));
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      if (!ring.piece(k)) continue;
      F2 f[4];
      unpack(r[k], f);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = f[e] * (inv_r * w_pre[k][e]);
      p.n_out[at + k * p.tpr] = pack(f);
    }
  }
}

template <int kVec, bool kFull>
__global__ void __launch_bounds__(kNormMostThreads)
block_norm_backward_kernel(const NormParams p) {
  extern __shared__ __align__(16) unsigned char smem_dyn[];
  float* joined = reinterpret_cast<float*>(smem_dyn);   // behind the last row: [rows][2H + 8], where a CTA takes several rows at a time
  __shared__ __align__(16) NormBuf buf[kBackwardRows][2];
  RowSums row_sums(buf, p.tpr);
  const int row_in = threadIdx.x / p.tpr, c0 = threadIdx.x % p.tpr, nv = p.H / 8;
  const float inv_h = 1.f / (float)p.H;
  pdl_prologue_done();
  F2 w_post[kVec][4], w_pre[kVec][4], sum_post[kVec][4], sum_pre[kVec][4];
  double sum_scale = 0.0;
#pragma unroll
  for (int k = 0; k < kVec; ++k) {
    if (c0 + k * p.tpr < nv) {
      load_gain(p.y != nullptr ? p.w_post : nullptr, c0 + k * p.tpr, w_post[k]);
      load_gain(p.d_n != nullptr ? p.w_pre : nullptr, c0 + k * p.tpr, w_pre[k]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sum_post[k][e] = sum_pre[k][e] = both(0.f);
  }
  const float scale = p.y != nullptr && p.scale != nullptr ? __ldg(p.scale) : 1.f;
  constexpr int kStages = kBackwardStages;
  const bool has_y = p.y != nullptr, has_n = p.d_n != nullptr, one_gate = has_y && p.gate_cols == 1, wide_gate = has_y && p.gate_cols > 1;
  const int step = (int)gridDim.x * p.rows;
  int row = (int)blockIdx.x * p.rows + row_in;
  const void* const arrays[5] = {has_n ? p.r : nullptr, p.d_n, p.d_r_out, p.y, wide_gate ? p.gate : nullptr};
  NormRing<kVec, kNormMostThreads, 5, kStages, kFull> ring(smem_dyn, p, row, c0);
  ring.clear(arrays);
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) ring.fetch(s, row + s * step < p.T, arrays);
  int stage = 0;
  float gate_next = one_gate && row < p.T ? bf16_bits_to_float(p.gate[row]) : 0.f;
  for (; row < p.T; row += step) {
    const size_t at = (size_t)row * nv + c0;
    float sg = 1.f, sg_rest = 0.f;
    if (one_gate) sg = sigmoid_of(gate_next, &sg_rest);
    if (one_gate && row + step < p.T) gate_next = bf16_bits_to_float(p.gate[row + step]);
    ring.fetch(stage == 0 ? kStages - 1 : stage - 1, row + (kStages - 1) * step < p.T, arrays);
    cp_async_wait<kStages - 1>();
    // sums of r^2, a r and y^2
    F2 s0 = both(0.f), s1 = s0, s2 = s0;
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      if (!ring.piece(k)) continue;
      F2 fr[4], fn[4], fy[4];
      unpack(ring.get(stage, 0, k), fr);
      unpack(ring.get(stage, 1, k), fn);
      unpack(ring.get(stage, 3, k), fy);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s0 = fma2(fr[e], fr[e], s0);
        s1 = fma2(fn[e] * w_pre[k][e], fr[e], s1);
        s2 = fma2(fy[e], fy[e], s2);
      }
    }
    float s[3] = {sum_of(s0), sum_of(s1), sum_of(s2)};
    row_sums(s);
    const float inv_r = rsqrtf(fmaf(s[0], inv_h, p.eps)), inv_y = p.normalise_y ? rsqrtf(fmaf(s[2], inv_h, p.eps)) : 1.f;
    // mean_h(a r_hat) / rms, taken times r_hat.  1 / rms goes in one factor at a time, each against one that is as large as rms: its cube alone leaves
    // fp32 at an rms of 1e-13 or 1e13, where the gradients do not.
    const F2 mean2 = both(-(inv_r * (inv_r * (s[1] * inv_h)))), inv_r2 = both(inv_r);
    const F2 post2 = both(scale * sg * inv_y);                  // what the products of d_r and y (and a channel's sigmoid) get in dw_post
    F2 f_dr[kVec][4];
    F2 q2[kVec];
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      q2[k] = both(0.f);
      if (!ring.piece(k)) continue;
      unpack(ring.get(stage, 2, k), f_dr[k]);
      F2 fr[4], fn[4];
      unpack(ring.get(stage, 0, k), fr);
      unpack(ring.get(stage, 1, k), fn);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const F2 r_hat = fr[e] * inv_r2;
        f_dr[k][e] = fma2(r_hat, mean2, fma2(fn[e] * inv_r2, w_pre[k][e], f_dr[k][e]));
        sum_pre[k][e] = fma2(fn[e], r_hat, sum_pre[k][e]);
      }
      if (p.d_r != nullptr) p.d_r[at + k * p.tpr] = pack(f_dr[k]);
      if (has_y) {
        F2 fy[4];
        unpack(ring.get(stage, 3, k), fy);
        if (wide_gate) {
          F2 g[4];
          unpack(ring.get(stage, 4, k), g);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const F2 t = f_dr[k][e] * fy[e] * sigmoid_of(g[e]);
            sum_post[k][e] = fma2(post2, t, sum_post[k][e]);
            q2[k] = fma2(t, w_post[k][e], q2[k]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const F2 t = f_dr[k][e] * fy[e];
            sum_post[k][e] = fma2(post2, t, sum_post[k][e]);
            q2[k] = fma2(t, w_post[k][e], q2[k]);
          }
        }
      }
    }
    const int stage_now = stage;
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (!has_y) continue;
    // With one gate a token its sigmoid is not in the products yet, nor is 1 / rms(y).  d_scale is a sum over the whole batch in which most cancels:
    // 64 bits beyond chains of four and one addition.
    if (kVec == 2) q2[0] = fma2(q2[kVec - 1], both(1.f), q2[0]);
    float q[2], q_factor = sg * inv_y;
    parts(q2[0], &q[0], &q[1]);
    sum_scale += (double)q_factor * ((double)q[0] + (double)q[1]);
    float q_sum[1] = {q_factor * (q[0] + q[1])};
    row_sums(q_sum);
    const float q_row = q_sum[0];
    if (c0 == 0 && one_gate && p.d_gate != nullptr) p.d_gate[row] = (uint16_t)(pack_bf16x2(scale * sg_rest * q_row, 0.f) & 0xFFFFu);
    if (p.d_y == nullptr && (p.d_gate == nullptr || !wide_gate)) continue;
    const F2 back2 = both(p.normalise_y ? -(inv_y * (scale * q_row * inv_h)) : 0.f), inv_y2 = both(inv_y);      // taken times y_hat
    const F2 out2 = both(inv_y * scale * sg);
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      if (!ring.piece(k)) continue;
      F2 fy[4], dy[4];
      unpack(ring.get(stage_now, 3, k), fy);
      if (wide_gate) {
        F2 g[4], dg[4];
        unpack(ring.get(stage_now, 4, k), g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float lo, hi, lo_rest, hi_rest;
          parts(g[e], &lo, &hi);
          lo = sigmoid_of(lo, &lo_rest);
          hi = sigmoid_of(hi, &hi_rest);
          const F2 b = w_post[k][e] * f_dr[k][e] * out2;
          dy[e] = fma2(b, pair_of(lo, hi), fy[e] * inv_y2 * back2);
          dg[e] = b * fy[e] * pair_of(lo * lo_rest, hi * hi_rest);
        }
        if (p.d_gate != nullptr) reinterpret_cast<uint4*>(p.d_gate)[at + k * p.tpr] = pack(dg);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) dy[e] = fma2(w_post[k][e] * f_dr[k][e], out2, fy[e] * inv_y2 * back2);
      }
      if (p.d_y != nullptr) p.d_y[at + k * p.tpr] = pack(dy);
    }
  }
  if (p.partial == nullptr) return;
  // the CTA's sums: its row groups one after the other
  sum_scale = row_sums(sum_scale);
  const size_t width = 2 * (size_t)p.H + 8;
  float* out = p.partial + (size_t)blockIdx.x * width;
  float* own = out;
  if (p.rows > 1) {
    cp_async_wait<0>();
    __syncthreads();                     // the ring's place is free
    own = joined + row_in * width;
  }
#pragma unroll
  for (int k = 0; k < kVec; ++k) {
    const int v = c0 + k * p.tpr;
    if (v >= nv) continue;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float4 a, b;
      parts(sum_post[k][2 * h], &a.x, &a.y);
      parts(sum_post[k][2 * h + 1], &a.z, &a.w);
      parts(sum_pre[k][2 * h], &b.x, &b.y);
      parts(sum_pre[k][2 * h + 1], &b.z, &b.w);
      reinterpret_cast<float4*>(own)[2 * v + h] = a;
      reinterpret_cast<float4*>(own + p.H)[2 * v + h] = b;
    }
  }
  if (c0 == 0) *reinterpret_cast<double*>(own + 2 * p.H) = sum_scale;
  if (p.rows == 1) return;
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
}

// Columns of the CTAs' partial sums: 32 columns a CTA, kJoinRows threads a column, joined in order.
__global__ void __launch_bounds__(32 * kJoinRows)
block_norm_join_kernel(const float* __restrict__ partial, int n, int H, float* dw_post, float* dw_pre, float* d_scale) {
  __shared__ double part[kJoinRows][33];
  const int c = blockIdx.x * 32 + threadIdx.x, g = threadIdx.y;
  const size_t width = 2 * (size_t)H + 8;
  pdl_prologue_done();
  double a = 0.0;
  if (c < 2 * H) {
    float v[5];                                  // 148 rows at most over 32 threads
#pragma unroll
    for (int u = 0; u < 5; ++u) v[u] = g + u * kJoinRows < n ? partial[(size_t)(g + u * kJoinRows) * width + c] : 0.f;
#pragma unroll
    for (int u = 0; u < 5; ++u) a += (double)v[u];
  } else if (c == 2 * H) {
    for (int i = g; i < n; i += kJoinRows) a += *reinterpret_cast<const double*>(partial + (size_t)i * width + c);
  }
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

constexpr size_t kMostNormSmem = 168 * 1024;      // 2 stages x 5 arrays x 2 pieces x 512 threads x 16 bytes: 160 KB

struct NormPlan { int vec, tpr, rows; unsigned grid; size_t smem; };

// Two pieces of 8 elements a thread, one where a warp holds the row with one (H 256).  512 threads an SM: forward in CTAs of 128 (rows
// below 128 threads share one), as many as these threads allow (H 2056 to 2560, 160 threads a row: three, but the ring's place, laid out for 512 threads
// above 128, lets two be resident, and the last 148 wait); backward in one CTA, whose rows' sums leave as one row of partial sums (148
// rows to join instead of 444), with fewer rows at a time where 148 CTAs would not all get one.
NormPlan plan_of(const moe_norm_shape* s, bool backward) {
  NormPlan n{};
  const int nv = s->H / 8;
  n.vec = nv > 32 ? 2 : 1;
  n.tpr = ((nv + n.vec - 1) / n.vec + 31) / 32 * 32;
  if (backward) {
    const int fit = kNormMostThreads / n.tpr < kBackwardRows ? kNormMostThreads / n.tpr : kBackwardRows, wanted = (s->T + 147) / 148;
    n.rows = wanted < fit ? wanted : fit;
  } else {
    n.rows = n.tpr >= 128 ? 1 : 128 / n.tpr;
    if (n.rows > s->T) n.rows = s->T;
  }
  const int threads = n.tpr * n.rows, most = !backward && threads <= 128 ? 128 : kNormMostThreads;
  const long long ctas = ((long long)s->T + n.rows - 1) / n.rows, resident = 148ll * (backward ? 1 : kNormMostThreads / threads);
  n.grid = (unsigned)(ctas < resident ? ctas : resident);
  const int arrays = backward ? 5 : 3, stages = backward ? kBackwardStages : kForwardStages;
  n.smem = (size_t)stages * arrays * n.vec * most * 16;
  const size_t join = backward && n.rows > 1 ? n.rows * (2 * (size_t)s->H + 8) * sizeof(float) : 0;    // rows * H <= 8192: under 66 KB
  if (n.smem < join) n.smem = join;
  return n;
}

bool full_rows(const NormPlan& n, int H) { return n.tpr * n.vec * 8 == H; }      // every thread has all of its pieces

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
  static PerDeviceOnce once[5];
  const int which = n.vec == 1 ? 0 : (n.tpr * n.rows <= 128 ? 1 : 3) + full_rows(n, a.s->H);
  auto kernel = which == 0   ? block_norm_kernel<1, 128, false>
                : which == 1 ? block_norm_kernel<2, 128, false>
                : which == 2 ? block_norm_kernel<2, 128, true>
                : which == 3 ? block_norm_kernel<2, 512, false>
                             : block_norm_kernel<2, 512, true>;
  if (!ensure_dynamic_smem(kernel, kMostNormSmem, once[which])) return MOE_ERR_CUDA;
  return launch_dependent(kernel, dim3(n.grid), dim3((unsigned)(n.tpr * n.rows)), n.smem, a.stream, 1, p) == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

moe_status launch_block_norm_backward(const BlockNormArgs& a) {
  const NormPlan n = plan_of(a.s, true);
  NormParams p = params_of(a, n);
  const bool sums = a.dw_post != nullptr || a.dw_pre != nullptr || a.d_scale != nullptr;
  p.partial = sums ? static_cast<float*>(a.ws) : nullptr;
  static PerDeviceOnce once[3];
  const int which = n.vec == 1 ? 0 : 1 + full_rows(n, a.s->H);
  auto kernel = which == 0 ? block_norm_backward_kernel<1, false> : which == 1 ? block_norm_backward_kernel<2, false> : block_norm_backward_kernel<2, true>;
  if (!ensure_dynamic_smem(kernel, kMostNormSmem, once[which])) return MOE_ERR_CUDA;
  if (launch_dependent(kernel, dim3(n.grid), dim3((unsigned)(n.tpr * n.rows)), n.smem, a.stream, 1, p) != cudaSuccess) return MOE_ERR_CUDA;
  if (!sums) return MOE_OK;
  return launch_dependent(block_norm_join_kernel, dim3((unsigned)((2 * a.s->H + 1 + 31) / 32)), dim3(32, kJoinRows), 0, a.stream, 1,
                          static_cast<const float*>(p.partial), (int)n.grid, (int)a.s->H, a.dw_post, a.dw_pre, a.d_scale) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}
