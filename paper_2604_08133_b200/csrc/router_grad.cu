// Gradients of the router: the balance loss over the kept pairs, the backward pass of Eq. 1 (moe_gate) and the
// gradients of Eq. 2's weighted sum.  See include/allocmoe.h for the formulas.
#include "common.cuh"
#include "router_grad.h"

namespace allocmoe {

// ------------------------------------------------------------------------------------------------ packed sequences
// Bound b of the packed sequences, clamped to [0, T] (no offsets: one sequence of all T rows).
DEV int seq_bound(const int32_t* off, int b, int T) {
  return off == nullptr ? (b == 0 ? 0 : T) : min(max(__ldg(off + b), 0), T);
}

// Whole warp: the first sequence that ends behind row r (n_seq if none), i.e. the number of b with bound b+1 <= r.
// 32 probes per step; on offsets that are not monotone it still ends within [0, n_seq].
DEV int first_seq_behind(const int32_t* off, int n_seq, int T, int r) {
  const int lane = threadIdx.x & 31;
  int lo = 0, len = n_seq;
  while (len > 0) {
    const int step = (len + 31) / 32;
    const int b = lo + lane * step;
    const bool behind = lane * step < len && seq_bound(off, b + 1, T) <= r;
    const int k = __popc(__ballot_sync(0xffffffffu, behind));
    if (k == 0) break;
    const int end = min(lo + k * step, lo + len);
    lo += (k - 1) * step + 1;
    len = end - lo;
  }
  return lo;
}

// One thread: the sequence that holds row r, or -1 (n_seq >= 1).
DEV int seq_of_row(const int32_t* off, int n_seq, int T, int r) {
  if (off == nullptr) return 0;
  int lo = 0, hi = n_seq;   // bound lo <= r < bound hi once both ends are checked
  if (r < seq_bound(off, 0, T) || r >= seq_bound(off, n_seq, T)) return -1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (seq_bound(off, mid, T) <= r) lo = mid; else hi = mid;
  }
  return lo;
}

// ------------------------------------------------------------------------------------------------ balance loss
// Unit of work: a warp owns kBalRows consecutive rows and walks the sequences that overlap them.  A sequence that
// lies inside one warp's rows is finished there; of one that crosses a border every warp leaves a partial sum (slot
// 0: the sequence came in from earlier rows, slot 1: it starts here), and where all rows of a CTA belong to one
// sequence the CTA joins its warps' sums into one partial.  balance_finish joins the partials of each sequence in row
// order, so the bits do not depend on which CTA ran first; the counts are integers.
// Bound by reading the scores once (4 T N bytes) for long batches, by latency for short ones.
constexpr int kBalRows = 32;
constexpr int kBalWarps = 8;
constexpr int kBalThreads = 32 * kBalWarps;
constexpr int kBalCtaRows = kBalRows * kBalWarps;
constexpr int kMaxN = 128;

struct BalanceParams {
  const float* scores;
  const int32_t* topk_idx;
  const int32_t* n_sel;
  const int32_t* seq_offsets;
  int T, N, K, n_seq;
  float alpha;
  int32_t* counts;
  float* coef;
  float* loss;
  int32_t* dev_status;
  float* part_sum;      // [warps][2][N]
  int32_t* part_cnt;    // [warps][2][N]
  float* cta_sum;       // [ctas][N]
  int32_t* cta_cnt;     // [ctas][N]
  float* seq_loss;      // [n_seq]
  unsigned* ticket;     // CTAs of balance_finish_kernel that are done
};

struct BalanceSmem {
  float sum[kBalWarps][kMaxN];
  int cnt[kBalWarps][kMaxN];
  float tot[kMaxN];
  int itot[kMaxN];
  float wsum[kBalWarps];
  int flag;
};

DEV float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
DEV int warp_sum(int v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// alpha N c / (n_seq C T_b), the derivative of the loss with respect to every score of the expert in the sequence
DEV float balance_coef(const BalanceParams& p, int cnt, int C, int rows) {
  if (C <= 0) return 0.f;
  return (float)cnt / (float)C * (p.alpha * (float)p.N / (float)p.n_seq) / (float)rows;
}

// One warp: sums of the scores and counts of the kept pairs over rows [a, e), left in s.sum[warp] and s.cnt[warp].
template <int CG>   // lanes per row: N / 4 rounded up to 8, 16 or 32
DEV void balance_piece(const BalanceParams& p, BalanceSmem& s, int warp, int lane, int a, int e) {
  constexpr int kSubs = 32 / CG;
  const int sub = lane / CG, c = lane % CG;
  for (int i = lane; i < p.N; i += 32) s.cnt[warp][i] = 0;
  __syncwarp();
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  bool bad = false;
  if (4 * c < p.N) {
    const float* col = p.scores + 4 * c;
#pragma unroll 8
    for (int t = a + sub; t < e; t += kSubs) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(col + (size_t)t * p.N));
      // false for NaN, infinity and negative values
      bad |= !(v.x >= 0.f && v.y >= 0.f && v.z >= 0.f && v.w >= 0.f && v.x <= 3.4e38f && v.y <= 3.4e38f && v.z <= 3.4e38f &&
               v.w <= 3.4e38f);
      acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
    }
  }
#pragma unroll
  for (int d = CG; d < 32; d <<= 1) {
    acc.x += __shfl_xor_sync(0xffffffffu, acc.x, d);
    acc.y += __shfl_xor_sync(0xffffffffu, acc.y, d);
    acc.z += __shfl_xor_sync(0xffffffffu, acc.z, d);
    acc.w += __shfl_xor_sync(0xffffffffu, acc.w, d);
  }
  if (sub == 0 && 4 * c < p.N) *reinterpret_cast<float4*>(&s.sum[warp][4 * c]) = acc;
  bool bad_id = false;
  const int pairs = (e - a) * p.K;
  for (int q = lane; q < pairs; q += 32) {
    const int t = a + q / p.K, j = q % p.K;
    const int n = p.n_sel == nullptr ? p.K : __ldg(p.n_sel + t);
    const int id = __ldg(p.topk_idx + (size_t)t * p.K + j);
    if (j < n) {
      if ((unsigned)id < (unsigned)p.N) atomicAdd(&s.cnt[warp][id], 1); else bad_id = true;
    }
  }
  if (bad) set_dev_status(p.dev_status, MOE_ERR_NONFINITE);
  if (bad_id) set_dev_status(p.dev_status, MOE_ERR_ARG);
  __syncwarp();
}

// A CTA whose rows all belong to one sequence (and are more than one warp's) leaves one partial for all of them.
DEV bool balance_cta_joined(int cta, int lo, int hi, int T) {
  const int r0 = cta * kBalCtaRows, r1 = min(r0 + kBalCtaRows, T);
  return lo <= r0 && hi >= r1 && r1 - r0 > kBalRows;
}

// Sequence b, rows [lo, hi) that cross a warp's border: joins its partials and writes its outputs.  Whole CTA.
DEV void balance_finish_seq(const BalanceParams& p, BalanceSmem& s, int b, int lo, int hi) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cols = p.N <= 32 ? 32 : (p.N <= 64 ? 64 : 128);
  const int groups = kBalThreads / cols, grp = tid / cols, col = tid % cols;
  const int w0 = lo / kBalRows, w1 = (hi - 1) / kBalRows, c0 = w0 / kBalWarps, c1 = w1 / kBalWarps;
  const bool j0 = balance_cta_joined(c0, lo, hi, p.T), j1 = balance_cta_joined(c1, lo, hi, p.T);
  const int n_head = j0 ? 0 : min(c0 * kBalWarps + kBalWarps - 1, w1) - w0 + 1;
  const int first_mid = j0 ? c0 : c0 + 1, last_mid = j1 ? c1 : c1 - 1;
  const int n_mid = max(last_mid - first_mid + 1, 0);
  const int n_tail = (c1 != c0 && !j1) ? w1 - c1 * kBalWarps + 1 : 0;
  const int n_all = n_head + n_mid + n_tail;
  float sum = 0.f;
  int cnt = 0;
  if (col < p.N) {
#pragma unroll 4
    for (int i = grp; i < n_all; i += groups) {
      const float* ps;
      const int32_t* pc;
      if (i >= n_head && i < n_head + n_mid) {
        const size_t at = (size_t)(first_mid + i - n_head) * p.N + col;
        ps = p.cta_sum + at;
        pc = p.cta_cnt + at;
      } else {
        const int w = i < n_head ? w0 + i : c1 * kBalWarps + (i - n_head - n_mid);
        const size_t at = ((size_t)w * 2 + (lo < w * kBalRows ? 0 : 1)) * p.N + col;
        ps = p.part_sum + at;
        pc = p.part_cnt + at;
      }
      sum += __ldcg(ps);
      cnt += __ldcg(pc);
    }
  }
  __syncthreads();   // the buffers below may still be read by the previous sequence's last step
  if (col < p.N) { s.sum[grp][col] = sum; s.cnt[grp][col] = cnt; }
  __syncthreads();
  if (tid < p.N) {
    for (int g = 1; g < groups; ++g) { sum += s.sum[g][tid]; cnt += s.cnt[g][tid]; }
    s.tot[tid] = sum;
    s.itot[tid] = cnt;
  }
  __syncthreads();
  if (warp == 0) {
    int C = 0;
    for (int i = lane; i < p.N; i += 32) C += s.itot[i];
    C = warp_sum(C);
    float term = 0.f;
    for (int i = lane; i < p.N; i += 32) {
      const float k = balance_coef(p, s.itot[i], C, hi - lo);
      p.counts[(size_t)b * p.N + i] = s.itot[i];
      p.coef[(size_t)b * p.N + i] = k;
      term = fmaf(k, s.tot[i], term);
    }
    term = warp_sum(term);
    if (lane == 0) p.seq_loss[b] = term;
  }
}

// The loss from the sequences' terms, in a fixed order.  Whole CTA.
DEV void balance_total(const BalanceParams& p, BalanceSmem& s) {
  float v = 0.f;
  for (int b = threadIdx.x; b < p.n_seq; b += kBalThreads) v += __ldcg(p.seq_loss + b);
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) s.wsum[threadIdx.x >> 5] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    float t = 0.f;
    for (int w = 0; w < kBalWarps; ++w) t += s.wsum[w];
    *p.loss = t;
  }
}

template <int CG>
__global__ void __launch_bounds__(kBalThreads)
balance_partial_kernel(const BalanceParams p) {
  __shared__ __align__(16) BalanceSmem s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_prologue_done();
  if (blockIdx.x == 0 && tid == 0) *p.ticket = 0u;

  // every sequence once, over all warps: offsets in order, outputs of the empty ones
  for (int b = blockIdx.x * kBalWarps + warp; b < p.n_seq; b += gridDim.x * kBalWarps) {
    if (p.seq_offsets != nullptr && lane == 0) {
      const int o0 = __ldg(p.seq_offsets + b), o1 = __ldg(p.seq_offsets + b + 1);
      if (o0 < 0 || o1 < o0 || o1 > p.T) set_dev_status(p.dev_status, MOE_ERR_ARG);
    }
    if (seq_bound(p.seq_offsets, b + 1, p.T) <= seq_bound(p.seq_offsets, b, p.T)) {
      for (int i = lane; i < p.N; i += 32) {
        p.counts[(size_t)b * p.N + i] = 0;
        p.coef[(size_t)b * p.N + i] = 0.f;
      }
      if (lane == 0) p.seq_loss[b] = 0.f;
    }
  }

  const int cr0 = blockIdx.x * kBalCtaRows;
  const int r0 = min(cr0 + warp * kBalRows, p.T), r1 = min(r0 + kBalRows, p.T);
  int b = first_seq_behind(p.seq_offsets, p.n_seq, p.T, cr0);
  const bool joined = b < p.n_seq && balance_cta_joined(blockIdx.x, seq_bound(p.seq_offsets, b, p.T),
                                                        seq_bound(p.seq_offsets, b + 1, p.T), p.T);
  if (joined) {
    if (r0 < r1) {
      balance_piece<CG>(p, s, warp, lane, r0, r1);
    } else {
      for (int i = lane; i < p.N; i += 32) { s.sum[warp][i] = 0.f; s.cnt[warp][i] = 0; }
    }
    __syncthreads();
    if (tid < p.N) {
      float sum = 0.f;
      int cnt = 0;
#pragma unroll
      for (int w = 0; w < kBalWarps; ++w) { sum += s.sum[w][tid]; cnt += s.cnt[w][tid]; }
      p.cta_sum[(size_t)blockIdx.x * p.N + tid] = sum;
      p.cta_cnt[(size_t)blockIdx.x * p.N + tid] = cnt;
    }
  } else if (r0 < r1) {
    b = first_seq_behind(p.seq_offsets, p.n_seq, p.T, r0);
    while (b < p.n_seq) {
      const int lo = seq_bound(p.seq_offsets, b, p.T), hi = seq_bound(p.seq_offsets, b + 1, p.T);
      if (lo >= r1) break;
      const int a = max(lo, r0), e = min(hi, r1);
      if (e > a) {
        balance_piece<CG>(p, s, warp, lane, a, e);
        if (lo >= r0 && hi <= r1) {   // the whole sequence
          int C = 0;
          for (int i = lane; i < p.N; i += 32) C += s.cnt[warp][i];
          C = warp_sum(C);
          float term = 0.f;
          for (int i = lane; i < p.N; i += 32) {
            const int cnt = s.cnt[warp][i];
            const float k = balance_coef(p, cnt, C, hi - lo);
            p.counts[(size_t)b * p.N + i] = cnt;
            p.coef[(size_t)b * p.N + i] = k;
            term = fmaf(k, s.sum[warp][i], term);
          }
          term = warp_sum(term);
          if (lane == 0) p.seq_loss[b] = term;
        } else {
          const size_t at = ((size_t)(r0 / kBalRows) * 2 + (lo < r0 ? 0 : 1)) * p.N;
          for (int i = lane; i < p.N; i += 32) {
            p.part_sum[at + i] = s.sum[warp][i];
            p.part_cnt[at + i] = s.cnt[warp][i];
          }
        }
        __syncwarp();
      }
      ++b;
      // a run of empty sequences is stepped over at once
      if (b < p.n_seq && seq_bound(p.seq_offsets, b + 1, p.T) <= hi) {
        const int next = first_seq_behind(p.seq_offsets, p.n_seq, p.T, hi);
        b = max(b, next);
      }
    }
  }
  if (gridDim.x == 1) {   // few rows: the same CTA joins the partials
    __syncthreads();
    for (int q = 0; q < p.n_seq; ++q) {
      const int lo = seq_bound(p.seq_offsets, q, p.T), hi = seq_bound(p.seq_offsets, q + 1, p.T);
      if (hi > lo && lo / kBalRows != (hi - 1) / kBalRows) balance_finish_seq(p, s, q, lo, hi);
    }
    __syncthreads();
    balance_total(p, s);
  }
}

// Joins the partials of the sequences that cross a warp's border, a CTA per sequence; the last CTA to finish sums the
// sequences' terms (its order is fixed, whichever CTA that is).
__global__ void __launch_bounds__(kBalThreads)
balance_finish_kernel(const BalanceParams p) {
  __shared__ __align__(16) BalanceSmem s;
  pdl_prologue_done();
  for (int b = blockIdx.x; b < p.n_seq; b += gridDim.x) {
    const int lo = seq_bound(p.seq_offsets, b, p.T), hi = seq_bound(p.seq_offsets, b + 1, p.T);
    if (hi > lo && lo / kBalRows != (hi - 1) / kBalRows) balance_finish_seq(p, s, b, lo, hi);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();   // seq_loss of this CTA's sequences, written by this thread
    s.flag = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (s.flag) balance_total(p, s);
}

// ------------------------------------------------------------------------------------------------ gate backward
// d_logits: a row on CG lanes, four experts a lane.  The row's softmax gradient needs one sum over the experts,
// taken by shuffles.  Bound by reading the scores and writing d_logits (8 T N bytes).
struct LogitGradParams {
  const float* scores;
  const int32_t* topk_idx;
  const int32_t* n_sel;
  const float* d_topk_score;
  const float* coef;
  const int32_t* seq_offsets;
  int T, N, K, n_seq;
  float* d_logits;
  int32_t* dev_status;
};
constexpr int kLgWarps = 8;

template <int CG>
__global__ void __launch_bounds__(32 * kLgWarps)
logit_grad_kernel(const LogitGradParams p) {
  constexpr int kSubs = 32 / CG;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int sub = lane / CG, c = lane % CG;
  pdl_prologue_done();
  if (p.seq_offsets != nullptr)
    for (int b = blockIdx.x * blockDim.x + threadIdx.x; b < p.n_seq; b += gridDim.x * blockDim.x) {
      const int o0 = __ldg(p.seq_offsets + b), o1 = __ldg(p.seq_offsets + b + 1);
      if (o0 < 0 || o1 < o0 || o1 > p.T) set_dev_status(p.dev_status, MOE_ERR_ARG);
    }
  const bool col_ok = 4 * c < p.N;
  const long long step = (long long)gridDim.x * kLgWarps * kSubs;
  // the loop's bound is the warp's first row, so that all lanes take part in the shuffles
  for (long long t0 = ((long long)blockIdx.x * kLgWarps + warp) * kSubs; t0 < p.T; t0 += step) {
    const int t = (int)t0 + sub;
    const int b = t < p.T ? seq_of_row(p.seq_offsets, p.n_seq, p.T, t) : -1;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f), g = v;
    if (b >= 0 && col_ok) {
      v = __ldg(reinterpret_cast<const float4*>(p.scores + (size_t)t * p.N + 4 * c));
      if (p.coef != nullptr) g = __ldg(reinterpret_cast<const float4*>(p.coef + (size_t)b * p.N + 4 * c));
      if (p.d_topk_score != nullptr) {
        const int n = p.n_sel == nullptr ? p.K : min(__ldg(p.n_sel + t), p.K);
        for (int j = 0; j < n; ++j) {
          const int id = __ldg(p.topk_idx + (size_t)t * p.K + j);
          const float d = __ldg(p.d_topk_score + (size_t)t * p.K + j);
          if ((unsigned)id >= (unsigned)p.N) { if (c == 0) set_dev_status(p.dev_status, MOE_ERR_ARG); }
          else if (id >> 2 == c) {
            const int k = id & 3;
            if (k == 0) g.x += d; else if (k == 1) g.y += d; else if (k == 2) g.z += d; else g.w += d;
          }
        }
      }
    }
    float dot = v.x * g.x + v.y * g.y + v.z * g.z + v.w * g.w;
#pragma unroll
    for (int d = CG / 2; d >= 1; d >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, d);
    if (t < p.T && col_ok) {
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      if (b >= 0) o = make_float4(v.x * (g.x - dot), v.y * (g.y - dot), v.z * (g.z - dot), v.w * (g.w - dot));
      *reinterpret_cast<float4*>(p.d_logits + (size_t)t * p.N + 4 * c) = o;
    }
  }
}

// dx[t] = d_logits[t] W_gate^T: a CTA per token.
__global__ void __launch_bounds__(256)
gate_dx_kernel(const float* __restrict__ d_logits, const uint16_t* __restrict__ W_gate, int H, int N, __nv_bfloat16* __restrict__ dx) {
  __shared__ float dl[kMaxN];
  pdl_prologue_done();
  const size_t t = blockIdx.x;
  for (int i = threadIdx.x; i < N; i += blockDim.x) dl[i] = d_logits[t * N + i];
  __syncthreads();
  for (int h = threadIdx.x; h < H; h += blockDim.x) {
    float acc = 0.f;
    for (int i = 0; i < N; i += 4) {
      const uint2 w = __ldg(reinterpret_cast<const uint2*>(W_gate + (size_t)h * N + i));
      acc = fmaf(dl[i], bf16_bits_to_float(w.x & 0xFFFFu), acc);
      acc = fmaf(dl[i + 1], bf16_bits_to_float(w.x >> 16), acc);
      acc = fmaf(dl[i + 2], bf16_bits_to_float(w.y & 0xFFFFu), acc);
      acc = fmaf(dl[i + 3], bf16_bits_to_float(w.y >> 16), acc);
    }
    dx[t * H + h] = __float2bfloat16_rn(acc);
  }
}

// Partial dW of one run of tokens: CTA = 64 rows of dW x all N experts, a thread per row and quarter of the experts.
__global__ void __launch_bounds__(256)
gate_dw_kernel(const float* __restrict__ d_logits, const uint16_t* __restrict__ x, const int32_t* __restrict__ seq_offsets,
               int n_seq, int T, int H, int N, int tokens_per_split, float* __restrict__ part, float* __restrict__ bias_part) {
  __shared__ float dl[kMaxN];
  pdl_prologue_done();
  const int h = blockIdx.x * 64 + (threadIdx.x & 63), q = threadIdx.x >> 6;
  const int n4 = N / 4, i0 = q * n4;
  int t0 = blockIdx.y * tokens_per_split, t1 = min(t0 + tokens_per_split, T);
  t0 = max(t0, seq_bound(seq_offsets, 0, T));          // rows of padding carry no gradient and are not read
  t1 = min(t1, seq_bound(seq_offsets, n_seq, T));
  float acc[kMaxN / 4];
#pragma unroll
  for (int i = 0; i < kMaxN / 4; ++i) acc[i] = 0.f;
  float bias = 0.f;
  for (int t = t0; t < t1; ++t) {
    __syncthreads();
    if (threadIdx.x < N) {
      dl[threadIdx.x] = d_logits[(size_t)t * N + threadIdx.x];
      bias += dl[threadIdx.x];
    }
    __syncthreads();
    const float xv = bf16_bits_to_float(x == nullptr ? 0u : (uint32_t)__ldg(x + (size_t)t * H + h));
#pragma unroll
    for (int i = 0; i < kMaxN / 4; ++i)
      if (i < n4) acc[i] = fmaf(xv, dl[i0 + i], acc[i]);
  }
  float* out = part + ((size_t)blockIdx.y * H + h) * N + i0;
#pragma unroll
  for (int i = 0; i < kMaxN / 4; ++i)
    if (i < n4) out[i] = acc[i];
  if (blockIdx.x == 0 && threadIdx.x < N) bias_part[(size_t)blockIdx.y * N + threadIdx.x] = bias;
}

__global__ void __launch_bounds__(256)
gate_dw_join_kernel(const float* __restrict__ part, const float* __restrict__ bias_part, int splits, int HN, int N,
                    float* __restrict__ dW, float* __restrict__ d_bias) {
  pdl_prologue_done();
  for (int i = blockIdx.x * 256 + threadIdx.x; i < HN; i += gridDim.x * 256) {
    float v = 0.f;
    for (int s = 0; s < splits; ++s) v += part[(size_t)s * HN + i];
    if (dW != nullptr) dW[i] = v;
  }
  if (d_bias != nullptr && blockIdx.x == 0 && threadIdx.x < N) {
    float v = 0.f;
    for (int s = 0; s < splits; ++s) v += bias_part[(size_t)s * N + threadIdx.x];
    d_bias[threadIdx.x] = v;
  }
}

// ------------------------------------------------------------------------------------------------ combine backward
// A CTA per token; warp j takes column j, j + 8: the dot product of d_out[t] with the pair's row of y_perm and, where
// asked for, the row topk_score * d_out[t].  Bound by bytes: y_perm and d_y_perm once, d_out once.
__global__ void __launch_bounds__(256)
combine_backward_kernel(const uint4* __restrict__ d_out, const uint4* __restrict__ y_perm, const int32_t* __restrict__ pair_pos,
                        const float* __restrict__ topk_score, const int32_t* __restrict__ n_sel, int K_orig, int row_vec,
                        long long budget, float* __restrict__ d_topk_score, uint4* __restrict__ d_y_perm) {
  const size_t t = blockIdx.x;
  const int lane = threadIdx.x & 31;
  pdl_prologue_done();
  const int n = min(__ldg(n_sel + t), K_orig);
  for (int j = threadIdx.x >> 5; j < K_orig; j += 8) {
    const int pos = __ldg(pair_pos + t * K_orig + j);
    float dot = 0.f;
    if (j < n && pos >= 0 && pos < budget) {
      const float w = d_y_perm != nullptr ? __ldg(topk_score + t * K_orig + j) : 0.f;
      for (int c = lane; c < row_vec; c += 32) {
        const uint4 a = __ldg(d_out + t * row_vec + c), y = __ldg(y_perm + (size_t)pos * row_vec + c);
        const uint32_t au[4] = {a.x, a.y, a.z, a.w}, yu[4] = {y.x, y.y, y.z, y.w};
        uint32_t o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float a0 = bf16_bits_to_float(au[q] & 0xFFFFu), a1 = bf16_bits_to_float(au[q] >> 16);
          dot = fmaf(a0, bf16_bits_to_float(yu[q] & 0xFFFFu), dot);
          dot = fmaf(a1, bf16_bits_to_float(yu[q] >> 16), dot);
          o[q] = pack_bf16x2(w * a0, w * a1);
        }
        if (d_y_perm != nullptr) d_y_perm[(size_t)pos * row_vec + c] = make_uint4(o[0], o[1], o[2], o[3]);
      }
      dot = warp_sum(dot);
    }
    if (lane == 0) d_topk_score[t * K_orig + j] = dot;
  }
}

}  // namespace allocmoe

using namespace allocmoe;

namespace {

// Carve-up of the router workspace; regions start on 256-byte boundaries.
struct RouterWs {
  size_t part_sum, part_cnt, cta_sum, cta_cnt, seq_loss, ticket;   // moe_balance_loss
  size_t d_logits, dw_part, bias_part;                             // moe_gate_backward
  size_t total;
};

int dw_splits(const moe_shape* s) {
  const int by_rows = (s->T + 127) / 128, by_sms = (2 * 148 * 64 + s->H - 1) / s->H;
  int n = by_rows < by_sms ? by_rows : by_sms;
  return n < 1 ? 1 : n;
}

RouterWs router_ws(const moe_shape* s, int n_seq) {
  RouterWs w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += (bytes + 255) & ~(size_t)255;
    return at;
  };
  const size_t ctas = ((size_t)s->T + kBalCtaRows - 1) / kBalCtaRows, N = s->N, H = s->H, sp = dw_splits(s);
  w.part_sum = take(ctas * kBalWarps * 2 * N * 4);
  w.part_cnt = take(ctas * kBalWarps * 2 * N * 4);
  w.cta_sum = take(ctas * N * 4);
  w.cta_cnt = take(ctas * N * 4);
  w.seq_loss = take((size_t)n_seq * 4);
  w.ticket = take(4);
  w.d_logits = take((size_t)s->T * N * 4);
  w.dw_part = take(sp * H * N * 4);
  w.bias_part = take(sp * N * 4);
  w.total = off;
  return w;
}

template <typename T>
T* in_ws(void* ws, size_t off) { return reinterpret_cast<T*>(static_cast<unsigned char*>(ws) + off); }

}  // namespace

size_t router_workspace_bytes(const moe_shape* s, int32_t n_seq) { return router_ws(s, n_seq).total; }

moe_status launch_balance_loss(const moe_shape* s, const float* scores, const int32_t* topk_idx, const int32_t* n_sel,
                               const int32_t* seq_offsets, int n_seq, float alpha, int32_t* counts, float* coef,
                               float* loss, int32_t* dev_status, void* ws, cudaStream_t stream) {
  const RouterWs w = router_ws(s, n_seq);
  BalanceParams p{};
  p.scores = scores;
  p.topk_idx = topk_idx;
  p.n_sel = n_sel;
  p.seq_offsets = seq_offsets;
  p.T = s->T;
  p.N = s->N;
  p.K = s->K_orig;
  p.n_seq = n_seq;
  p.alpha = alpha;
  p.counts = counts;
  p.coef = coef;
  p.loss = loss;
  p.dev_status = dev_status;
  p.part_sum = in_ws<float>(ws, w.part_sum);
  p.part_cnt = in_ws<int32_t>(ws, w.part_cnt);
  p.cta_sum = in_ws<float>(ws, w.cta_sum);
  p.cta_cnt = in_ws<int32_t>(ws, w.cta_cnt);
  p.seq_loss = in_ws<float>(ws, w.seq_loss);
  p.ticket = in_ws<unsigned>(ws, w.ticket);
  const unsigned ctas = (unsigned)(((long long)s->T + kBalCtaRows - 1) / kBalCtaRows);
  auto kernel = s->N <= 32 ? balance_partial_kernel<8> : s->N <= 64 ? balance_partial_kernel<16> : balance_partial_kernel<32>;
  if (launch_dependent(kernel, dim3(ctas), dim3(kBalThreads), 0, stream, 1, p) != cudaSuccess) return MOE_ERR_CUDA;
  if (ctas == 1) return MOE_OK;
  const unsigned fin = (unsigned)(n_seq < 148 ? n_seq : 148);
  return launch_dependent(balance_finish_kernel, dim3(fin), dim3(kBalThreads), 0, stream, 1, p) == cudaSuccess ? MOE_OK
                                                                                                               : MOE_ERR_CUDA;
}

moe_status launch_gate_backward(const GateBackwardArgs& a) {
  const moe_shape* s = a.s;
  const RouterWs w = router_ws(s, a.n_seq);
  LogitGradParams p{};
  p.scores = a.scores;
  p.topk_idx = a.topk_idx;
  p.n_sel = a.n_sel;
  p.d_topk_score = a.d_topk_score;
  p.coef = a.coef;
  p.seq_offsets = a.seq_offsets;
  p.T = s->T;
  p.N = s->N;
  p.K = s->K_orig;
  p.n_seq = a.n_seq;
  p.d_logits = a.d_logits != nullptr ? a.d_logits : in_ws<float>(a.ws, w.d_logits);
  p.dev_status = a.dev_status;
  const int cg = s->N <= 32 ? 8 : s->N <= 64 ? 16 : 32;
  const long long rows_per_cta = (long long)kLgWarps * (32 / cg);
  const long long want = (s->T + rows_per_cta - 1) / rows_per_cta;
  const unsigned ctas = (unsigned)(want < 148 * 8 ? want : 148 * 8);
  auto kernel = cg == 8 ? logit_grad_kernel<8> : cg == 16 ? logit_grad_kernel<16> : logit_grad_kernel<32>;
  if (launch_dependent(kernel, dim3(ctas), dim3(32 * kLgWarps), 0, a.stream, 1, p) != cudaSuccess) return MOE_ERR_CUDA;
  if (a.dx != nullptr &&
      launch_dependent(gate_dx_kernel, dim3((unsigned)s->T), dim3(256), 0, a.stream, 1, (const float*)p.d_logits, a.W_gate,
                       (int)s->H, (int)s->N, reinterpret_cast<__nv_bfloat16*>(a.dx)) != cudaSuccess)
    return MOE_ERR_CUDA;
  if (a.dW != nullptr || a.d_bias != nullptr) {
    const int splits = dw_splits(s);
    const int per = (s->T + splits - 1) / splits;
    float* part = in_ws<float>(a.ws, w.dw_part);
    float* bias_part = in_ws<float>(a.ws, w.bias_part);
    if (launch_dependent(gate_dw_kernel, dim3((unsigned)(s->H / 64), (unsigned)splits), dim3(256), 0, a.stream, 1,
                         (const float*)p.d_logits, a.x, a.seq_offsets, a.n_seq, (int)s->T, (int)s->H, (int)s->N, per, part,
                         bias_part) != cudaSuccess)
      return MOE_ERR_CUDA;
    if (launch_dependent(gate_dw_join_kernel, dim3(148 * 2), dim3(256), 0, a.stream, 1, (const float*)part,
                         (const float*)bias_part, splits, (int)(s->H * s->N), (int)s->N, a.dW, a.d_bias) != cudaSuccess)
      return MOE_ERR_CUDA;
  }
  return MOE_OK;
}

moe_status launch_combine_backward(const moe_shape* s, const uint16_t* d_out, const uint16_t* y_perm,
                                   const int32_t* pair_pos, const float* topk_score, const int32_t* n_sel,
                                   int64_t budget, float* d_topk_score, uint16_t* d_y_perm, cudaStream_t stream) {
  return launch_dependent(combine_backward_kernel, dim3((unsigned)s->T), dim3(256), 0, stream, 1,
                          reinterpret_cast<const uint4*>(d_out), reinterpret_cast<const uint4*>(y_perm), pair_pos, topk_score,
                          n_sel, (int)s->K_orig, s->H / 8, (long long)budget, d_topk_score,
                          reinterpret_cast<uint4*>(d_y_perm)) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}
