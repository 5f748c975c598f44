// Gradients of the router: the balance loss over the kept pairs, the backward pass of Eq. 1 (moe_gate) and the
// gradients of Eq. 2's weighted sum.  See include/allocmoe.h for the formulas.
#include <cooperative_groups.h>
#include <cuda.h>

#include "common.cuh"
#include "router_grad.h"
#include "tmap.h"

namespace cg = cooperative_groups;

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
// Unit of work: a warp owns 32 consecutive rows (4 where sequences are short, see bal_row_shift) and walks the sequences that overlap them.  A sequence that
// lies inside one warp's rows is finished there; of one that crosses a border every warp leaves a partial sum (slot
// 0: the sequence came in from earlier rows, slot 1: it starts here), and where all rows of a CTA belong to one
// sequence the CTA joins its warps' sums into one partial.  balance_finish joins the partials of each sequence in row
// order, so the bits do not depend on which CTA ran first; the counts are integers.
// Bound by reading the scores once (4 T N bytes) for long batches, by latency for short ones: a row's ids are read by one
// lane and counted by atomics in shared memory, the scores with eight 16-byte loads a lane in flight.  65 521 rows of 64
// experts in 37 sequences, from HBM: this and logit_grad_kernel together 26.6 us (their 35 MB at 1.3 TB/s: three launches one
// after the other, each with its own first loads and drain); 64 rows: 7.7 us, two launches.
constexpr int kBalWarps = 8;
constexpr int kBalThreads = 32 * kBalWarps;
constexpr int kMaxN = 128;
// Up to this many sequences of few rows are joined by the one CTA, more by a second launch (256 rows in 4 sequences 10 us either
// way, in 15 23 us and 13 us; in one 5 us by one launch).
constexpr int kBalOneCtaSeqs = 4;

struct BalanceParams {
  const float* scores;
  const int32_t* topk_idx;
  const int32_t* n_sel;
  const int32_t* seq_offsets;
  int T, N, K, n_seq;
  int row_shift;        // log2 of a warp's rows
  bool one_cta;         // balance_partial_kernel joins the partials and sums the loss itself
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
  unsigned top = 0u;   // largest bit pattern: above the largest finite value for NaN, infinity and anything negative
  if (4 * c < p.N) {
    const float* col = p.scores + 4 * c;
    for (int t = a + sub; t < e; t += 8 * kSubs) {   // eight rows' loads in flight a lane
      float4 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[i] = t + i * kSubs < e ? __ldg(reinterpret_cast<const float4*>(col + (size_t)(t + i * kSubs) * p.N)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // adding 0 makes a negative zero a positive one
        top = max(max(top, __float_as_uint(v[i].x + 0.f)), __float_as_uint(v[i].y + 0.f));
        top = max(max(top, __float_as_uint(v[i].z + 0.f)), __float_as_uint(v[i].w + 0.f));
        acc.x += v[i].x; acc.y += v[i].y; acc.z += v[i].z; acc.w += v[i].w;
      }
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
  for (int t = a + lane; t < e; t += 32) {   // a row a lane, the loads of eight of its columns in flight
    const int n = p.n_sel == nullptr ? p.K : min(__ldg(p.n_sel + t), p.K);
    const int32_t* idx = p.topk_idx + (size_t)t * p.K;
    for (int j0 = 0; j0 < n; j0 += 8) {
      int id[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) id[i] = j0 + i < n ? __ldg(idx + j0 + i) : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (j0 + i < n) {
          if ((unsigned)id[i] < (unsigned)p.N) atomicAdd(&s.cnt[warp][id[i]], 1); else bad_id = true;
        }
    }
  }
  if (top > 0x7F7FFFFFu) set_dev_status(p.dev_status, MOE_ERR_NONFINITE);
  if (bad_id) set_dev_status(p.dev_status, MOE_ERR_ARG);
  __syncwarp();
}

// A CTA whose rows all belong to one sequence (and are more than one warp's) leaves one partial for all of them.
DEV bool balance_cta_joined(const BalanceParams& p, int cta, int lo, int hi) {
  const int rows = kBalWarps << p.row_shift, r0 = cta * rows, r1 = min(r0 + rows, p.T);
  return lo <= r0 && hi >= r1 && r1 - r0 > rows / kBalWarps;
}
DEV bool balance_crosses(const BalanceParams& p, int lo, int hi) {   // a sequence that more than one warp has rows of
  return hi > lo && lo >> p.row_shift != (hi - 1) >> p.row_shift;
}

// The partials of a sequence whose rows are [lo, hi), in row order: warps' of the first CTA, CTAs', warps' of the last CTA.
struct BalanceParts {
  int w0, n_head, first_mid, n_mid, w_tail, n_all;
};
DEV BalanceParts balance_parts(const BalanceParams& p, int lo, int hi) {
  const int w0 = lo >> p.row_shift, w1 = (hi - 1) >> p.row_shift, c0 = w0 / kBalWarps, c1 = w1 / kBalWarps;
  const bool j0 = balance_cta_joined(p, c0, lo, hi), j1 = balance_cta_joined(p, c1, lo, hi);
  BalanceParts q;
  q.w0 = w0;
  q.n_head = j0 ? 0 : min(c0 * kBalWarps + kBalWarps - 1, w1) - w0 + 1;
  q.first_mid = j0 ? c0 : c0 + 1;
  q.n_mid = max((j1 ? c1 : c1 - 1) - q.first_mid + 1, 0);
  q.w_tail = c1 * kBalWarps;
  q.n_all = q.n_head + q.n_mid + ((c1 != c0 && !j1) ? w1 - q.w_tail + 1 : 0);
  return q;
}
DEV void balance_part_at(const BalanceParams& p, const BalanceParts& q, int lo, int i, const float** sum, const int32_t** cnt) {
  if (i >= q.n_head && i < q.n_head + q.n_mid) {
    const size_t at = (size_t)(q.first_mid + i - q.n_head) * p.N;
    *sum = p.cta_sum + at;
    *cnt = p.cta_cnt + at;
  } else {
    const int w = i < q.n_head ? q.w0 + i : q.w_tail + (i - q.n_head - q.n_mid);
    const size_t at = ((size_t)w * 2 + (lo < w << p.row_shift ? 0 : 1)) * p.N;
    *sum = p.part_sum + at;
    *cnt = p.part_cnt + at;
  }
}

// Sequence b, rows [lo, hi) that cross a warp's border: joins its partials and writes its outputs.  Whole CTA.
DEV void balance_finish_seq(const BalanceParams& p, BalanceSmem& s, int b, int lo, int hi) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cols = p.N <= 32 ? 32 : (p.N <= 64 ? 64 : 128);
  const int groups = kBalThreads / cols, grp = tid / cols, col = tid % cols;
  const BalanceParts q = balance_parts(p, lo, hi);
  float sum = 0.f;
  int cnt = 0;
  if (col < p.N) {
#pragma unroll 4
    for (int i = grp; i < q.n_all; i += groups) {
      const float* ps;
      const int32_t* pc;
      balance_part_at(p, q, lo, i, &ps, &pc);
      sum += __ldcg(ps + col);
      cnt += __ldcg(pc + col);
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

// The same by one warp, four experts a lane, for a sequence of few partials.
DEV void balance_finish_short(const BalanceParams& p, int b, int lo, int hi) {
  const int n0 = (threadIdx.x & 31) * 4;
  const BalanceParts q = balance_parts(p, lo, hi);
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  int4 cnt = make_int4(0, 0, 0, 0);
  if (n0 < p.N) {
#pragma unroll 4
    for (int i = 0; i < q.n_all; ++i) {
      const float* ps;
      const int32_t* pc;
      balance_part_at(p, q, lo, i, &ps, &pc);
      const float4 f = __ldcg(reinterpret_cast<const float4*>(ps + n0));
      const int4 c = __ldcg(reinterpret_cast<const int4*>(pc + n0));
      sum.x += f.x; sum.y += f.y; sum.z += f.z; sum.w += f.w;
      cnt.x += c.x; cnt.y += c.y; cnt.z += c.z; cnt.w += c.w;
    }
  }
  const int C = warp_sum(cnt.x + cnt.y + cnt.z + cnt.w);
  float term = 0.f;
  if (n0 < p.N) {
    const float4 k = make_float4(balance_coef(p, cnt.x, C, hi - lo), balance_coef(p, cnt.y, C, hi - lo),
                                 balance_coef(p, cnt.z, C, hi - lo), balance_coef(p, cnt.w, C, hi - lo));
    *reinterpret_cast<int4*>(p.counts + (size_t)b * p.N + n0) = cnt;
    *reinterpret_cast<float4*>(p.coef + (size_t)b * p.N + n0) = k;
    term = fmaf(k.x, sum.x, fmaf(k.y, sum.y, fmaf(k.z, sum.z, k.w * sum.w)));
  }
  term = warp_sum(term);
  if ((threadIdx.x & 31) == 0) p.seq_loss[b] = term;
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

  const int cr0 = min(((int)blockIdx.x * kBalWarps) << p.row_shift, p.T), w_all = blockIdx.x * kBalWarps + warp;
  const int r0 = min(w_all << p.row_shift, p.T), r1 = min(r0 + (1 << p.row_shift), p.T);
  int b = first_seq_behind(p.seq_offsets, p.n_seq, p.T, cr0);
  const bool joined = b < p.n_seq && balance_cta_joined(p, blockIdx.x, seq_bound(p.seq_offsets, b, p.T),
                                                        seq_bound(p.seq_offsets, b + 1, p.T));
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
          const size_t at = ((size_t)w_all * 2 + (lo < r0 ? 0 : 1)) * p.N;
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
  if (p.one_cta) {
    __syncthreads();
    for (int q = 0; q < p.n_seq; ++q) {
      const int lo = seq_bound(p.seq_offsets, q, p.T), hi = seq_bound(p.seq_offsets, q + 1, p.T);
      if (balance_crosses(p, lo, hi)) balance_finish_seq(p, s, q, lo, hi);
    }
    __syncthreads();
    balance_total(p, s);
  }
}

// Joins the partials of the sequences that cross a warp's border: a CTA per sequence; where there are more than CTAs, a warp
// per sequence of at most kBalShort partials (4096 sequences of 16 rows 76 -> 37 us; one of 4096 rows 8 us by a CTA, 13 us by
// a warp).  The last CTA to finish sums the sequences' terms (its order is fixed, whichever CTA that is).
constexpr int kBalShort = 16;
__global__ void __launch_bounds__(kBalThreads)
balance_finish_kernel(const BalanceParams p) {
  __shared__ __align__(16) BalanceSmem s;
  __shared__ int3 list[kBalThreads];   // sequence and rows: a warp's from the front, a CTA's from the back
  __shared__ int n_short, n_long;
  const int tid = threadIdx.x;
  pdl_prologue_done();
  for (int base = blockIdx.x; base < p.n_seq; base += gridDim.x * kBalThreads) {   // a sequence a thread
    if (tid == 0) n_short = n_long = 0;
    __syncthreads();
    const int b = base + tid * (int)gridDim.x;
    if (b < p.n_seq) {
      const int lo = seq_bound(p.seq_offsets, b, p.T), hi = seq_bound(p.seq_offsets, b + 1, p.T);
      if (balance_crosses(p, lo, hi)) {
        const bool is_short = p.n_seq > (int)gridDim.x && balance_parts(p, lo, hi).n_all <= kBalShort;
        const int at = is_short ? atomicAdd(&n_short, 1) : kBalThreads - 1 - atomicAdd(&n_long, 1);
        list[at] = make_int3(b, lo, hi);
      }
    }
    __syncthreads();
    for (int i = tid >> 5; i < n_short; i += kBalWarps) balance_finish_short(p, list[i].x, list[i].y, list[i].z);
    if ((tid & 31) == 0 && (tid >> 5) < n_short) __threadfence();   // seq_loss, written by this thread
    for (int i = 0; i < n_long; ++i) {
      const int3 q = list[kBalThreads - 1 - i];
      balance_finish_seq(p, s, q.x, q.y, q.z);
    }
    __syncthreads();
  }
  if (tid == 0) {
    __threadfence();   // seq_loss of the long sequences, written by this thread
    s.flag = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (s.flag) balance_total(p, s);
}

// ------------------------------------------------------------------------------------------------ gate backward
// Two launches.  logit_grad_kernel: d_logits, a row on CG lanes, four experts a lane; the softmax gradient needs one
// sum over the row's experts, taken by shuffles.  Where dx or dW is wanted it also writes d_logits as three bf16 terms
// (hi | mid | lo, NP = 4 CG columns each, zero beyond N and in rows of padding; together d_logits within 2^-24, an
// infinite value all in hi), the operand of both products, and for d_bias each CTA's column sums.  Bound by reading the
// scores and writing the results (8 N bytes a row and 6 NP for the terms: 64 with 8 experts, 160 with their terms) for long
// batches, else by its chain of dependent loads (offsets, coef, row).  Consecutive rows a warp and not strided ones: the
// sequence's offsets and coef are looked up once per run of rows.
struct LogitGradParams {
  const float* scores;
  const int32_t* topk_idx;
  const int32_t* n_sel;
  const float* d_topk_score;
  const float* coef;
  const int32_t* seq_offsets;
  int T, N, K, n_seq, H, rows_per_warp;
  float* d_logits;           // [T][N] or nullptr
  __nv_bfloat16* terms;      // [T][kTerms NP] or nullptr
  float* bias_part;          // [CTAs][N] or nullptr
  const uint16_t* W_gate;    // copied with rows of NP columns to w_pad where TMA cannot read it (N % 8 != 0)
  uint16_t* w_pad;           // [H][NP] or nullptr
  int32_t* dev_status;
};
constexpr int kLgWarps = 8;
constexpr int kTerms = 3;
constexpr int kNotKept = -1, kBadId = -2;   // in place of an expert id: a column that is not kept, an id outside [0, N)

template <int CG>
__global__ void __launch_bounds__(32 * kLgWarps)
logit_grad_kernel(const LogitGradParams p) {
  constexpr int kSubs = 32 / CG, NP = 4 * CG, kPer = CG >= 16 ? 1 : 16 / CG;   // kPer: pairs a lane holds (K <= 16)
  __shared__ __align__(16) float s_bias[kLgWarps][NP];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int sub = lane / CG, c = lane % CG;
  pdl_wait();                 // in this order: the second launch may read x and W_gate as soon as it starts
  pdl_launch_dependents();
  const bool col_ok = 4 * c < p.N;
  if (p.w_pad != nullptr)
    for (long long h = ((long long)blockIdx.x * kLgWarps + warp) * kSubs + sub; h < p.H; h += (long long)gridDim.x * kLgWarps * kSubs) {
      uint2 w = make_uint2(0u, 0u);
      if (col_ok) w = __ldg(reinterpret_cast<const uint2*>(p.W_gate + (size_t)h * p.N + 4 * c));
      *reinterpret_cast<uint2*>(p.w_pad + (size_t)h * NP + 4 * c) = w;
    }
  float4 bias = make_float4(0.f, 0.f, 0.f, 0.f);
  // A warp takes consecutive rows, so that the sequence it is in and its coef stay in registers; the next rows' loads are
  // on their way while the present ones are worked on.
  const long long first = ((long long)blockIdx.x * kLgWarps + warp) * p.rows_per_warp;
  const int begin = (int)min(first, (long long)p.T), end = (int)min(first + p.rows_per_warp, (long long)p.T);
  float4 v_next = make_float4(0.f, 0.f, 0.f, 0.f);
  int id_next[kPer];         // the kept pairs: lane c of the row holds columns c, c + CG, ...
  float d_next[kPer];
  auto fetch = [&](int t) {
    v_next = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int q = 0; q < kPer; ++q) { id_next[q] = kNotKept; d_next[q] = 0.f; }
    if (t >= end) return;
    if (col_ok) v_next = __ldg(reinterpret_cast<const float4*>(p.scores + (size_t)t * p.N + 4 * c));
    if (p.d_topk_score != nullptr) {
      const int n = p.n_sel == nullptr ? p.K : __ldg(p.n_sel + t);
#pragma unroll
      for (int q = 0; q < kPer; ++q) {
        const int j = c + q * CG;
        if (j < p.K) {
          const int i = __ldg(p.topk_idx + (size_t)t * p.K + j);
          const float f = __ldg(p.d_topk_score + (size_t)t * p.K + j);
          if (j < n) { id_next[q] = (unsigned)i < (unsigned)p.N ? i : kBadId; d_next[q] = f; }
        }
      }
    }
  };
  fetch(begin + sub);
  if (p.seq_offsets != nullptr)
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < p.n_seq; i += gridDim.x * blockDim.x) {
      const int o0 = __ldg(p.seq_offsets + i), o1 = __ldg(p.seq_offsets + i + 1);
      if (o0 < 0 || o1 < o0 || o1 > p.T) set_dev_status(p.dev_status, MOE_ERR_ARG);
    }
  int b = -1, seq_lo = 0, seq_hi = 0;
  float4 coef = make_float4(0.f, 0.f, 0.f, 0.f);
  // the loop's bound is the warp's first row, so that all lanes take part in the searches and shuffles
  for (int t0 = begin; t0 < end; t0 += kSubs) {
    const int t = t0 + sub;
    const bool row_ok = t < end;
    float4 v = v_next, g;
    int id[kPer];
    float d[kPer];
#pragma unroll
    for (int q = 0; q < kPer; ++q) { id[q] = id_next[q]; d[q] = d_next[q]; }
    fetch(t + kSubs);
    if (__any_sync(0xffffffffu, row_ok && (t < seq_lo || t >= seq_hi))) {   // another sequence, or padding
      b = first_seq_behind(p.seq_offsets, p.n_seq, p.T, t0);
      if (!row_ok || b >= p.n_seq) {
        b = -1;
      } else if (t < seq_bound(p.seq_offsets, b, p.T) || t >= seq_bound(p.seq_offsets, b + 1, p.T)) {
        b = seq_of_row(p.seq_offsets, p.n_seq, p.T, t);   // a later row of the warp's in a later sequence, or padding
      }
      seq_lo = b < 0 ? 0 : seq_bound(p.seq_offsets, b, p.T);
      seq_hi = b < 0 ? 0 : seq_bound(p.seq_offsets, b + 1, p.T);
      coef = make_float4(0.f, 0.f, 0.f, 0.f);
      if (b >= 0 && p.coef != nullptr && col_ok) coef = __ldg(reinterpret_cast<const float4*>(p.coef + (size_t)b * p.N + 4 * c));
    }
    g = coef;
    if (b < 0) v = make_float4(0.f, 0.f, 0.f, 0.f);     // padding may hold anything
    if (p.d_topk_score != nullptr) {
#pragma unroll
      for (int q = 0; q < kPer; ++q) {
        if (b >= 0 && id[q] == kBadId) set_dev_status(p.dev_status, MOE_ERR_ARG);
        const int first = q * CG, last = min(p.K, first + CG);
        for (int j = first; j < last; ++j) {
          const int i = __shfl_sync(0xffffffffu, id[q], sub * CG + j - first);
          const float f = __shfl_sync(0xffffffffu, d[q], sub * CG + j - first);
          if (b >= 0 && (i >> 2) == c) {   // never of a negative one
            const int k = i & 3;
            if (k == 0) g.x += f; else if (k == 1) g.y += f; else if (k == 2) g.z += f; else g.w += f;
          }
        }
      }
    }
    float dot = v.x * g.x + v.y * g.y + v.z * g.z + v.w * g.w;
#pragma unroll
    for (int d = CG / 2; d >= 1; d >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, d);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (b >= 0) o = make_float4(v.x * (g.x - dot), v.y * (g.y - dot), v.z * (g.z - dot), v.w * (g.w - dot));
    if (row_ok) {
      if (p.d_logits != nullptr && col_ok) *reinterpret_cast<float4*>(p.d_logits + (size_t)t * p.N + 4 * c) = o;
      if (p.terms != nullptr) {
        const uint2 hi = make_uint2(pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w));
        const float4 r1 = make_float4(bf16_rest(o.x, hi.x & 0xFFFFu), bf16_rest(o.y, hi.x >> 16),
                                      bf16_rest(o.z, hi.y & 0xFFFFu), bf16_rest(o.w, hi.y >> 16));
        const uint2 mid = make_uint2(pack_bf16x2(r1.x, r1.y), pack_bf16x2(r1.z, r1.w));
        const uint2 lo = make_uint2(pack_bf16x2(r1.x - bf16_bits_to_float(mid.x & 0xFFFFu), r1.y - bf16_bits_to_float(mid.x >> 16)),
                                    pack_bf16x2(r1.z - bf16_bits_to_float(mid.y & 0xFFFFu), r1.w - bf16_bits_to_float(mid.y >> 16)));
        uint2* row = reinterpret_cast<uint2*>(p.terms + (size_t)t * kTerms * NP);
        row[c] = hi;
        row[CG + c] = mid;
        row[2 * CG + c] = lo;
      }
      bias.x += o.x; bias.y += o.y; bias.z += o.z; bias.w += o.w;
    }
  }
  if (p.bias_part != nullptr) {
#pragma unroll
    for (int d = CG; d < 32; d <<= 1) {
      bias.x += __shfl_xor_sync(0xffffffffu, bias.x, d);
      bias.y += __shfl_xor_sync(0xffffffffu, bias.y, d);
      bias.z += __shfl_xor_sync(0xffffffffu, bias.z, d);
      bias.w += __shfl_xor_sync(0xffffffffu, bias.w, d);
    }
    if (sub == 0) *reinterpret_cast<float4*>(&s_bias[warp][4 * c]) = bias;
    __syncthreads();
    if (threadIdx.x < p.N) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kLgWarps; ++w) v += s_bias[w][threadIdx.x];
      p.bias_part[(size_t)blockIdx.x * p.N + threadIdx.x] = v;
    }
  }
}

// The sum of the CTAs' column sums, where neither product is wanted.  One CTA of 1024 threads.
__global__ void __launch_bounds__(1024)
bias_join_kernel(const float* __restrict__ bias_part, int parts, int N, float* __restrict__ d_bias) {
  __shared__ float s[8][kMaxN];
  pdl_prologue_done();
  const int n = threadIdx.x & (kMaxN - 1), g = threadIdx.x / kMaxN;
  float v = 0.f;
  if (n < N)
#pragma unroll 4
    for (int i = g; i < parts; i += 8) v += __ldg(bias_part + (size_t)i * N + n);
  s[g][n] = v;
  __syncthreads();
  if (threadIdx.x < N) {
#pragma unroll
    for (int q = 1; q < 8; ++q) v += s[q][n];
    d_bias[n] = v;
  }
}

// dx and dW in one pass over x and the terms of d_logits, on the tensor cores.  A CTA owns 128 columns of H (a
// slice) and a run of 128-token blocks.  Per block TMA brings x's 128 x 128 piece and the block's terms; both products
// read them where they lie:
//   dx[128 tokens, 128 h] = [hi | mid] [W W]^T       terms as the K-major A operand, W_gate's slice (resident) as B, twice
//   dW[128 h, terms]     += x^T [hi | mid | lo]      both as MN-major operands: the tokens are the K dimension
// dx is rounded to bf16, so two terms (2^-16 of d_logits) are enough there; dW stays fp32 and takes all three.  Up to 64
// experts the terms are columns of one product and are added at the end; beyond that all add into the same columns.
// x is read once and dx written once (packed in shared memory, stored by TMA).  The tensor cores' accumulation truncates,
// so every kGbFlush blocks the epilogue warps add dW's columns to sums in registers and the product starts over.  The
// CTAs of a slice form a cluster and add their sums through distributed shared memory in rank order.  Rows of padding
// have zero terms; their x is set to zero in shared memory before the product (a NaN there would survive a zero).
// Bound by HBM: x in, dx out (4 T H bytes); the terms come from L2, once per slice.  With logit_grad_kernel, from HBM: 8192
// tokens of 4096, 8 experts 32.0 us (4.2 TB/s); 4099 tokens of 2048, 60 experts in 9 sequences 23.8 us (1.5 TB/s: 16 slices x 6
// = 96 CTAs, about 6 blocks each, so the ring's filling, the flushes and the join weigh); 64 tokens 11.5 us (two launches and
// the join).  Plain loops on the CUDA cores took 1287, 465 and 65 us.
constexpr int kGbThreads = 320;                     // warp 0 TMA, 1 MMA, 2-9 epilogue
constexpr int kGbBlock = 128;                       // tokens per block
constexpr int kGbSlice = 128;                       // columns of H per CTA
constexpr int kGbBox = kGbBlock * 64 * 2;           // 16 KB: 64 columns x 128 rows
constexpr int kGbMaxStages = 3;
constexpr int kGbMaxCluster = 6;                    // 132 CTAs of this size are resident in clusters of 6, 120 in clusters of 8
constexpr int kGbFlush = 4;

template <int NP>
struct GbCfg {
  static constexpr int kTermBoxes = (kTerms * NP + 63) / 64;             // 1, 2, 3, 6
  static constexpr int kDwCols = NP <= 64 ? kTerms * NP : NP;            // 48, 96, 192, 128
  static constexpr int kWBoxes = NP <= 64 ? 1 : 2;
  static constexpr int kStageBytes = (2 + kTermBoxes) * kGbBox;
  static constexpr int kStages = NP == 16 ? 3 : NP <= 64 ? 2 : 1;        // 144, 128, 160, 128 KB
  static constexpr size_t kSmem = (size_t)kStages * kStageBytes + (kWBoxes + 2) * kGbBox + 1024;
};

struct GbParams {
  const int32_t* seq_offsets;
  int n_seq, T, H, N, blocks;
  bool want_dx;
  float* dW;                  // or nullptr
  float* d_bias;              // or nullptr
  const float* bias_part;
  int bias_parts;
  bool w_is_input;            // W_gate itself, not the copy that the first launch makes
  int32_t* dev_status;
};

struct GbCtl {
  uint64_t full[kGbMaxStages], empty[kGbMaxStages], w_full, dx_full[2], dx_empty[2], dw_full, dw_empty, drain;
  uint32_t tmem_base;
  volatile int abort_flag;
  float bias[kMaxN];
};

template <int NP>
__global__ void __launch_bounds__(kGbThreads, 1)
gate_products_kernel(const GbParams p, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_t,
                     const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_dx) {
  using C = GbCfg<NP>;
  cg::cluster_group cluster = cg::this_cluster();
  const int splits = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
  unsigned char* w_tile = ring + C::kStages * C::kStageBytes;
  unsigned char* out_tile = w_tile + C::kWBoxes * kGbBox;   // dx, 4 KB per epilogue warp
  __shared__ GbCtl ctl;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h0 = blockIdx.x * kGbSlice;
  if (tid == 0) {
    for (int s = 0; s < C::kStages; ++s) { mbar_init(&ctl.full[s], 1); mbar_init(&ctl.empty[s], 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(&ctl.dx_full[a], 1); mbar_init(&ctl.dx_empty[a], 8); }
    mbar_init(&ctl.w_full, 1);
    mbar_init(&ctl.dw_full, 1);
    mbar_init(&ctl.dw_empty, 8);
    mbar_init(&ctl.drain, 1);
    ctl.abort_flag = 0;
    fence_barrier_init();
    prefetch_tensormap(&tm_x);
    prefetch_tensormap(&tm_t);
    prefetch_tensormap(&tm_w);
    prefetch_tensormap(&tm_dx);
  }
  if (warp == 1) {
    tmem_alloc(&ctl.tmem_base, 512);
    tmem_relinquish();
  }
  pdl_launch_dependents();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = ctl.tmem_base;
  const uint32_t tmem_dw = tmem + 256;                 // dx: two accumulators of 128 columns, then dW
  volatile int* abort_flag = &ctl.abort_flag;
  const bool want_dx = p.want_dx, want_dw = p.dW != nullptr;
  // rows that carry a gradient, and this CTA's blocks
  const int row_lo = seq_bound(p.seq_offsets, 0, p.T), row_hi = seq_bound(p.seq_offsets, p.n_seq, p.T);
  const int per = (p.blocks + splits - 1) / splits;
  const int b0 = min(rank * per, p.blocks), b1 = min(b0 + per, p.blocks);
  auto has_rows = [&](int b) { return want_dw && b * kGbBlock < row_hi && (b + 1) * kGbBlock > row_lo; };
  auto flush_after = [&](int b) { return want_dw && ((b - b0) % kGbFlush == kGbFlush - 1 || b == b1 - 1); };
  constexpr int kSumCols = NP < 32 ? 16 : NP / 2;      // epilogue warps: dW of one row of the slice, half of the experts
  float sum[kSumCols];                                 // (all of them where that is less than a read of 16 columns)
#pragma unroll
  for (int i = 0; i < kSumCols; ++i) sum[i] = 0.f;
  const int q = warp & 3, half = (warp - 2) >> 2;      // epilogue warps: TMEM lanes, column half
  const bool sums = kSumCols * half < NP;

  if (warp == 0) {
    if (elect_one()) {
      if (want_dx && b0 < b1) {
        if (!p.w_is_input) pdl_wait();
        mbar_expect_tx(&ctl.w_full, C::kWBoxes * kGbBox);
        for (int i = 0; i < C::kWBoxes; ++i) tma_load_2d(w_tile + i * kGbBox, &tm_w, &ctl.w_full, i * 64, h0);
      }
      int it = 0;
      for (int b = b0; b < b1; ++b, ++it) {
        const int s = it % C::kStages;
        if (!mbar_wait_bounded(&ctl.empty[s], ((it / C::kStages) & 1u) ^ 1u, abort_flag, p.dev_status, kWaitLimitClk)) break;
        unsigned char* st = ring + s * C::kStageBytes;
        const bool x_too = has_rows(b);
        mbar_expect_tx(&ctl.full[s], (uint32_t)((x_too ? 2 : 0) + C::kTermBoxes) * kGbBox);
        if (x_too) {
          tma_load_2d(st, &tm_x, &ctl.full[s], h0, b * kGbBlock);
          tma_load_2d(st + kGbBox, &tm_x, &ctl.full[s], h0 + 64, b * kGbBlock);
        }
        if (it == 0) pdl_wait();
        for (int i = 0; i < C::kTermBoxes; ++i) tma_load_2d(st + (2 + i) * kGbBox, &tm_t, &ctl.full[s], i * 64, b * kGbBlock);
      }
      for (int k = it > C::kStages ? it - C::kStages : 0; k < it; ++k) mbar_wait_drain(&ctl.full[k % C::kStages], (k / C::kStages) & 1u);
      if (want_dx && b0 < b1) mbar_wait_drain(&ctl.w_full, 0u);
    }
  } else if (warp == 1) {
    constexpr uint32_t idesc_dx = umma_idesc_bf16(kGbBlock, kGbSlice);
    constexpr uint32_t idesc_dw = umma_idesc_bf16(kGbSlice, C::kDwCols) | (1u << 15) | (1u << 16);   // A and B MN-major
    const bool lead = elect_one();
    bool ok = true, dw_begun = false;
    if (want_dx && b0 < b1) ok = mbar_spin_bounded_warp(&ctl.w_full, 0u, abort_flag, p.dev_status, kWaitLimitClk);
    int it = 0, flushes = 0;
    for (int b = b0; ok && b < b1; ++b, ++it) {
      const int s = it % C::kStages;
      if (!(ok = mbar_spin_bounded_warp(&ctl.full[s], (it / C::kStages) & 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
      unsigned char* st = ring + s * C::kStageBytes;
      const uint32_t sx = smem_u32(st), stm = sx + 2 * kGbBox;
      if (want_dx) {
        const int a = it & 1;
        if (!(ok = mbar_spin_bounded_warp(&ctl.dx_empty[a], ((it >> 1) & 1u) ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
        tc_fence_after_sync();
        if (lead) {
          const uint32_t sw = smem_u32(w_tile);
#pragma unroll
          for (int k = 0; k < 2 * NP / 16; ++k) {
            const int ct = k * 16, cw = ct % NP;        // column among the terms, and in W
            const uint64_t da = umma_desc_sw128(stm + (ct / 64) * kGbBox) + (uint64_t)((ct % 64) * 2 / 16);
            const uint64_t db = umma_desc_sw128(sw + (cw / 64) * kGbBox) + (uint64_t)((cw % 64) * 2 / 16);
            umma_bf16(tmem + a * 128, da, db, idesc_dx, k != 0 ? 1u : 0u);
          }
          umma_commit(&ctl.dx_full[a]);
        }
      }
      if (want_dw && flushes > 0 && (b - b0) % kGbFlush == 0) {   // the sums of the blocks so far have been taken
        if (!(ok = mbar_spin_bounded_warp(&ctl.dw_empty, (flushes - 1) & 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
        dw_begun = false;
      }
      if (has_rows(b)) {
        const int t0 = b * kGbBlock;
        if (t0 < row_lo || min(t0 + kGbBlock, p.T) > row_hi) {   // rows of padding in this block
          for (int r = 0; r < kGbBlock; ++r) {
            if (t0 + r >= row_lo && t0 + r < row_hi) continue;
            if (lane < 16) *reinterpret_cast<uint4*>(st + (lane >> 3) * kGbBox + r * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async_smem();
          __syncwarp();
        }
        tc_fence_after_sync();
        if (lead) {
          const uint64_t da = umma_desc_mn_sw128(sx, kGbBox);
#pragma unroll
          for (int f = 0; f < kTerms * NP / C::kDwCols; ++f) {
            const uint64_t db = umma_desc_mn_sw128(stm + f * (C::kDwCols / 64) * kGbBox, kGbBox);
#pragma unroll
            for (int k = 0; k < kGbBlock / 16; ++k)
              umma_bf16(tmem_dw, da + (uint64_t)(k * (2048 >> 4)), db + (uint64_t)(k * (2048 >> 4)), idesc_dw,
                        (dw_begun || f != 0 || k != 0) ? 1u : 0u);
          }
        }
        dw_begun = true;
      }
      if (lead) umma_commit(&ctl.empty[s]);
      if (flush_after(b)) {
        if (lead) umma_commit(&ctl.dw_full);
        ++flushes;
      }
      __syncwarp();
    }
    if (lead) {                                          // every product of this CTA is complete
      umma_commit(&ctl.drain);
      mbar_wait_drain(&ctl.drain, 0u);
    }
    __syncwarp();
  } else {
    unsigned char* mine = out_tile + (warp - 2) * 4096;  // 32 rows x 64 columns, 128-byte swizzle
    int it = 0, flushes = 0;
    bool ok = true, any = false;
    for (int b = b0; ok && b < b1; ++b, ++it) {
      if (want_dx) {
        const int a = it & 1;
        if (!(ok = mbar_spin_bounded_warp(&ctl.dx_full[a], (it >> 1) & 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
        tc_fence_after_sync();
        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(a * 128 + half * 64);
        uint32_t u[2][32];
        tmem_ld_32x32(taddr, u[0]);
        tmem_ld_32x32(taddr + 32, u[1]);
        tmem_ld_wait();
        tc_fence_before_sync();
        if (lane == 0) {
          mbar_arrive(&ctl.dx_empty[a]);
          bulk_wait_read_all();                          // the previous block's tile has left
        }
        __syncwarp();
        const int t = b * kGbBlock + q * 32 + lane;
        if (t < row_lo || t >= row_hi) {                 // padding, whatever W_gate holds
#pragma unroll
          for (int k = 0; k < 32; ++k) u[0][k] = u[1][k] = 0u;
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t* w = &u[k / 4][(k % 4) * 8];
          *reinterpret_cast<uint4*>(mine + lane * 128 + ((k ^ (lane & 7)) << 4)) =
              make_uint4(pack_bf16x2(__uint_as_float(w[0]), __uint_as_float(w[1])), pack_bf16x2(__uint_as_float(w[2]), __uint_as_float(w[3])),
                         pack_bf16x2(__uint_as_float(w[4]), __uint_as_float(w[5])), pack_bf16x2(__uint_as_float(w[6]), __uint_as_float(w[7])));
        }
        fence_proxy_async_smem();
        __syncwarp();
        const int row = b * kGbBlock + q * 32, col = h0 + half * 64;
        if (lane == 0 && row < p.T && col < p.H) {
          tma_store_2d(mine, &tm_dx, col, row);
          bulk_commit();
        }
      }
      any |= has_rows(b);
      if (flush_after(b)) {
        if (!(ok = mbar_spin_bounded_warp(&ctl.dw_full, flushes & 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
        ++flushes;
        tc_fence_after_sync();
        if (any && sums) {
          constexpr int kSums = C::kDwCols / NP;         // terms side by side: smallest first
          const uint32_t taddr = tmem_dw + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * kSumCols);
#pragma unroll
          for (int c0 = 0; c0 < kSumCols; c0 += 16) {
            float v[16];
#pragma unroll
            for (int f = kSums - 1; f >= 0; --f) {
              uint32_t u[16];
              tmem_ld_32x16(taddr + (uint32_t)(f * NP + c0), u);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) v[i] = f == kSums - 1 ? __uint_as_float(u[i]) : v[i] + __uint_as_float(u[i]);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[c0 + i] += v[i];
          }
          tc_fence_before_sync();
        }
        any = false;
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.dw_empty);
      }
    }
    if (lane == 0) bulk_wait_all();
    __syncwarp();
  }
  if (p.d_bias != nullptr && blockIdx.x == 0) {
    // this rank's share of the column sums
    pdl_wait();
    const int share = (p.bias_parts + splits - 1) / splits;
    const int i0 = min(rank * share, p.bias_parts), i1 = min(i0 + share, p.bias_parts);
    if (tid < p.N) {
      float v = 0.f;
#pragma unroll 8
      for (int i = i0; i < i1; ++i) v += __ldcg(p.bias_part + (size_t)i * p.N + tid);
      ctl.bias[tid] = v;
    }
  }
  __syncthreads();                                       // the ring is free: every load landed, every product is complete
  float* part = reinterpret_cast<float*>(ring);
  const int RS = p.N + 1;
  if (want_dw && warp >= 2 && sums) {
    const bool aborted = ctl.abort_flag != 0;
#pragma unroll
    for (int i = 0; i < kSumCols; ++i) {
      const int n = half * kSumCols + i;
      if (n < p.N) part[(q * 32 + lane) * RS + n] = aborted ? __int_as_float(0x7fc00000) : sum[i];
    }
  }
  cluster.sync();
  if (want_dw) {
    const float* peer[kGbMaxCluster];
#pragma unroll
    for (int k = 0; k < kGbMaxCluster; ++k) peer[k] = cluster.map_shared_rank(part, k < splits ? k : 0);
    const int rows = min(kGbSlice, p.H - h0);
    for (int row = rank + splits * warp; row < rows; row += splits * (kGbThreads / 32))
      for (int n = lane; n < p.N; n += 32) {
        float v[kGbMaxCluster];
#pragma unroll
        for (int k = 0; k < kGbMaxCluster; ++k) v[k] = k < splits ? peer[k][row * RS + n] : 0.f;
#pragma unroll
        for (int k = 1; k < kGbMaxCluster; ++k) v[0] += v[k];
        p.dW[(size_t)(h0 + row) * p.N + n] = v[0];
      }
  }
  if (p.d_bias != nullptr && blockIdx.x == 0 && rank == 0 && tid < p.N) {
    float v = 0.f;
    for (int k = 0; k < splits; ++k) v += *cluster.map_shared_rank(&ctl.bias[tid], k);
    p.d_bias[tid] = v;
  }
  cluster.sync();   // no CTA leaves while a peer reads its sums
  pdl_wait();       // also where no role came to it: this launch ends after the one before it
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------------------------------------ combine backward
// A warp per (token, column): the dot product of d_out[t] with the pair's row of y_perm and, where asked for, the row
// topk_score * d_out[t], four 16-byte pieces a lane in flight.  Bound by bytes: y_perm and d_y_perm once, d_out once.  CTAs
// of two warps, so that the columns that are not kept free their slots at once, and the rows of y_perm and d_y_perm, each
// touched once, marked for early eviction, which keeps d_out (read once per kept pair) in L2.  4096 tokens, 12 288 pairs of
// 2048, inputs from HBM: 23.3 us (5.0 TB/s), 27.8 us with CTAs of eight warps; with the inputs partly in L2 19.5 us, 25.4 us
// without the marks.
constexpr int kCbWarps = 2;
constexpr int kCbBatch = 4;
__global__ void __launch_bounds__(32 * kCbWarps)
combine_backward_kernel(const uint4* __restrict__ d_out, const uint4* __restrict__ y_perm, const int32_t* __restrict__ pair_pos,
                        const float* __restrict__ topk_score, const int32_t* __restrict__ n_sel, int T, int K_orig, int row_vec,
                        long long budget, float* __restrict__ d_topk_score, uint4* __restrict__ d_y_perm) {
  const int lane = threadIdx.x & 31;
  pdl_prologue_done();
  const long long pair = (long long)blockIdx.x * kCbWarps + (threadIdx.x >> 5);
  if (pair >= (long long)T * K_orig) return;
  const size_t t = (size_t)(pair / K_orig);
  const int j = (int)(pair - (long long)t * K_orig);
  const int n = min(__ldg(n_sel + t), K_orig);
  const int pos = __ldg(pair_pos + t * K_orig + j);
  const float w = d_y_perm != nullptr ? __ldg(topk_score + t * K_orig + j) : 0.f;
  float dot = 0.f;
  if (j < n && pos >= 0 && pos < budget) {
    const uint4* a_row = d_out + t * row_vec;
    const uint4* y_row = y_perm + (size_t)pos * row_vec;
    uint4* y_out = d_y_perm + (size_t)pos * row_vec;
    for (int c = lane; c < row_vec; c += 32 * kCbBatch) {
      uint4 a[kCbBatch], y[kCbBatch];
#pragma unroll
      for (int k = 0; k < kCbBatch; ++k) {
        a[k] = y[k] = make_uint4(0u, 0u, 0u, 0u);
        if (c + 32 * k < row_vec) { y[k] = __ldcs(y_row + c + 32 * k); a[k] = __ldg(a_row + c + 32 * k); }
      }
#pragma unroll
      for (int k = 0; k < kCbBatch; ++k) {
        if (c + 32 * k >= row_vec) break;
        const uint32_t au[4] = {a[k].x, a[k].y, a[k].z, a[k].w}, yu[4] = {y[k].x, y[k].y, y[k].z, y[k].w};
        uint32_t o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float a0 = bf16_bits_to_float(au[q] & 0xFFFFu), a1 = bf16_bits_to_float(au[q] >> 16);
          dot = fmaf(a0, bf16_bits_to_float(yu[q] & 0xFFFFu), dot);
          dot = fmaf(a1, bf16_bits_to_float(yu[q] >> 16), dot);
          o[q] = pack_bf16x2(w * a0, w * a1);
        }
        if (d_y_perm != nullptr) __stcs(y_out + c + 32 * k, make_uint4(o[0], o[1], o[2], o[3]));
      }
    }
    dot = warp_sum(dot);
  }
  if (lane == 0) d_topk_score[t * K_orig + j] = dot;
}

}  // namespace allocmoe

using namespace allocmoe;

namespace {

// Carve-up of the router workspace; regions start on 256-byte boundaries.
struct RouterWs {
  size_t part_sum, part_cnt, cta_sum, cta_cnt, seq_loss, ticket;   // moe_balance_loss
  size_t terms, w_pad, bias_part;                                  // moe_gate_backward
  size_t total;
};

constexpr int kLgMaxCtas = 296;

int term_cols(int N) { return N <= 16 ? 16 : N <= 32 ? 32 : N <= 64 ? 64 : 128; }

// log2 of the rows a warp of balance_partial_kernel owns.  It walks their sequences one after the other, so 4 where they are
// shorter than 16 rows on average (64 sequences of one row 93 -> 16 us, 256 rows in 64 sequences 36 -> 8 us).
int bal_row_shift(int T, int n_seq) { return n_seq > 1 && (long long)n_seq * 16 >= T ? 2 : 5; }
long long bal_ctas(int T, int n_seq) {
  const int rows = kBalWarps << bal_row_shift(T, n_seq);
  return ((long long)T + rows - 1) / rows;
}

RouterWs router_ws(const moe_shape* s, int n_seq) {
  RouterWs w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += (bytes + 255) & ~(size_t)255;
    return at;
  };
  const size_t ctas = (size_t)bal_ctas(s->T, n_seq), N = s->N, NP = term_cols(s->N);
  w.part_sum = take(ctas * kBalWarps * 2 * N * 4);
  w.part_cnt = take(ctas * kBalWarps * 2 * N * 4);
  w.cta_sum = take(ctas * N * 4);
  w.cta_cnt = take(ctas * N * 4);
  w.seq_loss = take((size_t)n_seq * 4);
  w.ticket = take(4);
  w.terms = take((size_t)s->T * kTerms * NP * 2);
  w.w_pad = take(N % 8 != 0 ? (size_t)s->H * NP * 2 : 0);
  w.bias_part = take((size_t)kLgMaxCtas * N * 4);
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
  p.row_shift = bal_row_shift(s->T, n_seq);
  const unsigned ctas = (unsigned)bal_ctas(s->T, n_seq);
  auto kernel = s->N <= 32 ? balance_partial_kernel<8> : s->N <= 64 ? balance_partial_kernel<16> : balance_partial_kernel<32>;
  // few rows and sequences: one launch; else a warp per sequence for the empty ones, up to a CTA per SM
  p.one_cta = ctas == 1 && n_seq <= kBalOneCtaSeqs;
  const unsigned help = (unsigned)((n_seq + kBalWarps - 1) / kBalWarps), few = help < 148 ? help : 148, grid = ctas > few ? ctas : few;
  if (launch_dependent(kernel, dim3(grid), dim3(kBalThreads), 0, stream, 1, p) != cudaSuccess) return MOE_ERR_CUDA;
  if (p.one_cta) return MOE_OK;
  const unsigned fin = (unsigned)(n_seq < 148 ? n_seq : 148);
  return launch_dependent(balance_finish_kernel, dim3(fin), dim3(kBalThreads), 0, stream, 1, p) == cudaSuccess ? MOE_OK
                                                                                                               : MOE_ERR_CUDA;
}

namespace {

template <int NP>
moe_status launch_gate_products(const GateBackwardArgs& a, const GbParams& p, const void* terms, const void* W, int w_cols, int sms) {
  const moe_shape* s = a.s;
  CUtensorMap tm_x, tm_t, tm_w, tm_dx;
  // a map that nothing uses still has to be valid: the terms stand in for what was not given
  const bool has_x = a.dW != nullptr, has_w = a.dx != nullptr;
  if (!make_tmap(&tm_t, terms, kTerms * NP, (uint64_t)s->T, 0, kTerms * NP, 0, kGbBlock)) return MOE_ERR_CUDA;
  tm_x = tm_w = tm_dx = tm_t;
  if (has_x && !make_tmap(&tm_x, a.x, (uint64_t)s->H, (uint64_t)s->T, 0, (uint64_t)s->H, 0, kGbBlock)) return MOE_ERR_CUDA;
  if (has_w && !make_tmap(&tm_w, W, (uint64_t)w_cols, (uint64_t)s->H, 0, (uint64_t)w_cols, 0, kGbSlice)) return MOE_ERR_CUDA;
  if (has_w && !make_tmap(&tm_dx, a.dx, (uint64_t)s->H, (uint64_t)s->T, 0, (uint64_t)s->H, 0, 32)) return MOE_ERR_CUDA;
  static PerDeviceOnce attr_set;
  if (!ensure_dynamic_smem(gate_products_kernel<NP>, GbCfg<NP>::kSmem, attr_set)) return MOE_ERR_CUDA;
  // CTAs per slice: about one CTA per SM (each fills an SM's shared memory), every one with a block
  const int slices = (s->H + kGbSlice - 1) / kGbSlice;
  int splits = sms / slices;
  if (splits > p.blocks) splits = p.blocks;
  if (splits > kGbMaxCluster) splits = kGbMaxCluster;
  if (splits < 1) splits = 1;
  return launch_dependent(gate_products_kernel<NP>, dim3((unsigned)slices, (unsigned)splits), dim3(kGbThreads), GbCfg<NP>::kSmem,
                          a.stream, (unsigned)splits, p, tm_x, tm_t, tm_w, tm_dx) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}

}  // namespace

moe_status launch_gate_backward(const GateBackwardArgs& a) {
  const moe_shape* s = a.s;
  const RouterWs w = router_ws(s, a.n_seq);
  const bool products = a.dx != nullptr || a.dW != nullptr, pad = a.dx != nullptr && s->N % 8 != 0;
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
  p.H = s->H;
  p.d_logits = a.d_logits;
  p.terms = products ? in_ws<__nv_bfloat16>(a.ws, w.terms) : nullptr;
  p.bias_part = a.d_bias != nullptr ? in_ws<float>(a.ws, w.bias_part) : nullptr;
  p.W_gate = a.W_gate;
  p.w_pad = pad ? in_ws<uint16_t>(a.ws, w.w_pad) : nullptr;
  p.dev_status = a.dev_status;
  const int NP = term_cols(s->N), cg = NP / 4;
  const long long rows_per_cta = (long long)kLgWarps * (32 / cg);
  const long long want = (s->T + rows_per_cta - 1) / rows_per_cta;
  const int most = a.d_bias != nullptr ? kLgMaxCtas : 148 * 8;
  // rows per warp: a multiple of what it works on at a time, for about `most` CTAs
  const long long steps = (want + most - 1) / most;
  p.rows_per_warp = (int)steps * (32 / cg);
  const int ctas = (int)((want + steps - 1) / steps);
  auto kernel = cg == 4 ? logit_grad_kernel<4> : cg == 8 ? logit_grad_kernel<8> : cg == 16 ? logit_grad_kernel<16> : logit_grad_kernel<32>;
  if (launch_dependent(kernel, dim3((unsigned)ctas), dim3(32 * kLgWarps), 0, a.stream, 1, p) != cudaSuccess) return MOE_ERR_CUDA;
  if (products) {
    GbParams g{};
    g.seq_offsets = a.seq_offsets;
    g.n_seq = a.n_seq;
    g.T = s->T;
    g.H = s->H;
    g.N = s->N;
    g.blocks = (s->T + kGbBlock - 1) / kGbBlock;
    g.want_dx = a.dx != nullptr;
    g.dW = a.dW;
    g.d_bias = a.d_bias;
    g.bias_part = p.bias_part;
    g.bias_parts = ctas;
    g.w_is_input = !pad;
    g.dev_status = a.dev_status;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return MOE_ERR_CUDA;
    const void* W = pad ? (const void*)p.w_pad : (const void*)a.W_gate;
    const int w_cols = pad ? NP : s->N;
    if (NP == 16) return launch_gate_products<16>(a, g, p.terms, W, w_cols, sms);
    if (NP == 32) return launch_gate_products<32>(a, g, p.terms, W, w_cols, sms);
    if (NP == 64) return launch_gate_products<64>(a, g, p.terms, W, w_cols, sms);
    return launch_gate_products<128>(a, g, p.terms, W, w_cols, sms);
  }
  if (a.d_bias != nullptr)
    return launch_dependent(bias_join_kernel, dim3(1), dim3(1024), 0, a.stream, 1, (const float*)p.bias_part, ctas, (int)s->N,
                            a.d_bias) == cudaSuccess
               ? MOE_OK
               : MOE_ERR_CUDA;
  return MOE_OK;
}

moe_status launch_combine_backward(const moe_shape* s, const uint16_t* d_out, const uint16_t* y_perm,
                                   const int32_t* pair_pos, const float* topk_score, const int32_t* n_sel,
                                   int64_t budget, float* d_topk_score, uint16_t* d_y_perm, cudaStream_t stream) {
  return launch_dependent(combine_backward_kernel, dim3((unsigned)(((long long)s->T * s->K_orig + kCbWarps - 1) / kCbWarps)), dim3(32 * kCbWarps), 0, stream, 1,
                          reinterpret_cast<const uint4*>(d_out), reinterpret_cast<const uint4*>(y_perm), pair_pos, topk_score,
                          n_sel, (int)s->T, (int)s->K_orig, s->H / 8, (long long)budget, d_topk_score,
                          reinterpret_cast<uint4*>(d_y_perm)) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}
