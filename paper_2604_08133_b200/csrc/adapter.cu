// Projections with a low-rank adapter per request beside the shared weight:
//   v[t] = scale[a] x[t] A_a^T          (inner values, a = adapter_id[t])
//   y[t] = x[t] W^T + v[t] B_a^T
// and the same with SwiGLU over the pairs of output rows (the shared experts' first projection).
//
// Two launches.  The first computes the inner values; the second is the shared projection, which needs them only at
// the end of a tile and therefore starts while the first is still running.
//
// Few tokens (at most kDotTokens): every token reads its own adapter on the CUDA cores, in the first launch A, in the
// second B, beside the K loop.  Many tokens: both adapter products run on the tensor cores per block of tokens, over the
// adapters that the block's tokens name (its slots):
//   first launch   D = X [A_s0; A_s1; ...]^T, of which each token keeps its own slot's columns;
//   second launch  after a tile's K loop, for every slot one more K block [V masked to the slot's rows | B_slot].
// The inner values enter that product as two bf16 terms, v = hi + lo, 32 ranks a K block: hi in its first half, lo in its
// second, both against the same 32 columns of B.  bf16 is the operand type of the tensor cores beside a bf16 B; one term would
// round v to 2^-8, two leave 2^-16, below y's own rounding unless the terms cancel to less than 2^-8 of their size.  Where all tokens of a block name one adapter the block's V is loaded like
// any operand.  Elsewhere it is masked, and a zero in V times an infinity or NaN in B would reach the rows of other
// requests: the first launch looks through the B of such blocks' adapters, and an adapter with a non-finite value is left
// out of the products there; the epilogue adds its terms to its own rows.
#include <cooperative_groups.h>
#include <cuda.h>

#include "adapter.h"
#include "common.cuh"
#include "tmap.h"

namespace cg = cooperative_groups;

namespace allocmoe {

constexpr int kAM = 128;                       // tokens per tile (UMMA M)
constexpr int kABK = 64;                       // K per stage: one 128-byte swizzle row
constexpr int kAXBytes = kAM * kABK * 2;       // 16 KB
constexpr int kRankChunk = 32;                 // ranks per K block of the second adapter product
constexpr int kDotTokens = 128;

// The adapters named by the tokens of one block, in order of first appearance, and each token's place among them.
template <int kRows>
struct SlotList {
  int n;
  int uniform;           // the block's tokens all name the one adapter
  int pad[2];
  int adapter[kRows];
  int row_slot[kRows];   // -1: no adapter
};
constexpr int kPairM = 2 * kAM;   // tokens per tile of a CTA pair
constexpr int kBadParts = 16;     // at most two blocks of 128 tokens times a cluster of eight
typedef SlotList<kPairM> PairSlots;

struct AdapterParams {
  int T, K, M, n_adapters, rank, k_per_sub, swiglu_rows;
  const uint16_t* x;
  const uint16_t* A;
  const uint16_t* B;
  const float* scale;
  const int32_t* adapter_id;
  uint16_t* y;
  int32_t* dev_status;
  float* v;            // few tokens: [T][rank] inner values
  __nv_bfloat16* vt;   // many tokens: [T][rank chunks][hi 32 | lo 32]
  PairSlots* slots;    // [blocks of 256 tokens]
  unsigned* bad;       // [blocks of 256 tokens][kBadParts][8]: bit = slot, its B is not finite
  int parts;           // CTAs that look through the B of a block, per 128 tokens of it
};

DEV int valid_adapter(int a, int n) { return a < 0 || a >= n ? -1 : a; }

DEV float dot8(const uint4& a, const uint4& b, float acc) {
  const uint32_t au[4] = {a.x, a.y, a.z, a.w}, bu[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    acc = fmaf(bf16_bits_to_float(au[q] & 0xFFFFu), bf16_bits_to_float(bu[q] & 0xFFFFu), acc);
    acc = fmaf(bf16_bits_to_float(au[q] >> 16), bf16_bits_to_float(bu[q] >> 16), acc);
  }
  return acc;
}

// acc + the dot product of eight fp32 values and eight bf16 values
DEV float fma8f(const float4& v0, const float4& v1, const uint4& b, float s) {
  s = fmaf(v0.x, bf16_bits_to_float(b.x & 0xFFFFu), s);
  s = fmaf(v0.y, bf16_bits_to_float(b.x >> 16), s);
  s = fmaf(v0.z, bf16_bits_to_float(b.y & 0xFFFFu), s);
  s = fmaf(v0.w, bf16_bits_to_float(b.y >> 16), s);
  s = fmaf(v1.x, bf16_bits_to_float(b.z & 0xFFFFu), s);
  s = fmaf(v1.y, bf16_bits_to_float(b.z >> 16), s);
  s = fmaf(v1.z, bf16_bits_to_float(b.w & 0xFFFFu), s);
  return fmaf(v1.w, bf16_bits_to_float(b.w >> 16), s);
}

// A role's place in a ring of stages: the stage, the parity of its current use.
struct RingPos {
  int s = 0;
  uint32_t ph = 0;
  DEV void next(int stages) {
    if (++s == stages) { s = 0; ph ^= 1u; }
  }
  DEV void skip(int n, int stages) {   // n further
    s += n;
    ph ^= (uint32_t)(s / stages) & 1u;
    s %= stages;
  }
};

// ------------------------------------------------------------------------------------------------ inner values, few tokens
// A warp per token and kRows rows of its A.  Bound by reading the named adapters' A, at few tokens by the latency of one pass
// over K; times with the second launch, below.
template <int kRows>
__global__ void __launch_bounds__(256)
adapter_inner_dot_kernel(const AdapterParams p) {
  pdl_wait();                 // the second launch may read x and W as soon as it starts: everything before this is done
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int groups = p.rank / kRows;
  const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int t = (int)(unit / groups), r0 = (int)(unit % groups) * kRows;
  if (t >= p.T) return;
  const int id = __ldg(p.adapter_id + t);
  const int a = valid_adapter(id, p.n_adapters);
  if (a < 0) {
    if (id >= 0 && lane == 0 && r0 == 0) set_dev_status(p.dev_status, MOE_ERR_ARG);
    return;
  }
  const uint4* xr = reinterpret_cast<const uint4*>(p.x + (size_t)t * p.K);
  const uint4* ar = reinterpret_cast<const uint4*>(p.A + ((size_t)a * p.rank + r0) * p.K);
  const int nv = p.K / 8;
  float acc[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) acc[i] = 0.f;
#pragma unroll 4
  for (int c = lane; c < nv; c += 32) {
    const uint4 xv = __ldg(xr + c);
#pragma unroll
    for (int i = 0; i < kRows; ++i) acc[i] = dot8(xv, __ldg(ar + (size_t)i * nv + c), acc[i]);
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], d);
  }
  if (lane == 0) {
    const float s = __ldg(p.scale + a);
#pragma unroll
    for (int i = 0; i < kRows; ++i) p.v[(size_t)t * p.rank + r0 + i] = s * acc[i];
  }
}

DEV bool any_nonfinite(const uint4& w) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  bool bad = false;
#pragma unroll
  for (int k = 0; k < 4; ++k) bad |= (u[k] & 0x7F80u) == 0x7F80u || (u[k] & 0x7F800000u) == 0x7F800000u;
  return bad;
}

// ------------------------------------------------------------------------------------------------ inner values, many tokens
// A cluster of KS CTAs per block of 128 tokens and group of slots (as many as fill 256 columns), rank r of the cluster
// taking the 64-wide blocks r, r + KS, ... of K.  x and the slots' A rows come by TMA, tcgen05.mma (M 128, N = the
// group's columns) accumulates in TMEM, every token's own columns go to shared memory, and the ranks' partial sums are
// added in rank order through distributed shared memory.  The warps that have nothing to do meanwhile look through the B
// of a mixed block's adapters, each CTA of the block a part of it.
// Bound by latency: at 4096 tokens of K 2048, rank 64, 8 adapters 32 clusters of four, with the slot list, 8 K blocks a CTA and
// the join one after the other; a CTA fills an SM, so the second launch starts as these end.  Times with it, below.
constexpr int kInnerCols = 256;
constexpr int kInnerStageBytes = kAXBytes + kInnerCols * kABK * 2;   // 48 KB
constexpr int kInnerStages = 4;
constexpr int kInnerThreads = 256;

struct SlotScratch {
  int key[2 * kPairM], first[2 * kPairM];   // hash table: adapter, its first row; later (by row) the slot of a first row
  int warp_sums[33];
};

// Whole CTA of kInnerThreads >= kRows threads: the slot list of the kRows tokens from t0 on, in shared memory.  A hash
// table of twice as many places as tokens finds every adapter's first row (its place depends on the order of the inserts,
// the first row, a minimum, does not); one insert per warp and adapter.
template <int kRows>
DEV void build_slots(const AdapterParams& p, int t0, SlotList<kRows>* s, SlotScratch& h, bool report) {
  const int tid = threadIdx.x, lane = tid & 31;
  for (int i = tid; i < 2 * kPairM; i += kInnerThreads) {
    h.key[i] = -1;
    h.first[i] = kRows;
  }
  int id = -1;
  if (tid < kRows) {
    const int t = t0 + tid;
    const int raw = t < p.T ? __ldg(p.adapter_id + t) : -1;
    if (report && raw >= p.n_adapters) set_dev_status(p.dev_status, MOE_ERR_ARG);
    id = valid_adapter(raw, p.n_adapters);
  }
  __syncthreads();
  const unsigned same = __match_any_sync(0xffffffffu, id);
  const int leader = __ffs((int)same) - 1;
  int place = 0;
  if (id >= 0 && lane == leader) {
    place = (int)(((unsigned)id * 2654435761u) >> 16) & (2 * kPairM - 1);
    while (true) {
      const int old = atomicCAS(&h.key[place], -1, id);
      if (old == -1 || old == id) break;
      place = (place + 1) & (2 * kPairM - 1);
    }
    atomicMin(&h.first[place], tid);
  }
  place = __shfl_sync(0xffffffffu, place, leader);
  __syncthreads();
  const int f = id >= 0 ? h.first[place] : -1;   // the first row with the same adapter
  const bool is_first = f == tid;
  int n;
  const int slot = block_exclusive_scan(is_first ? 1 : 0, h.warp_sums, &n);
  if (is_first) {
    h.key[tid] = slot;
    s->adapter[slot] = id;
  }
  __syncthreads();
  const int mine = id >= 0 ? h.key[f] : -1;
  if (tid < kRows) s->row_slot[tid] = mine;
  const int all_first = __syncthreads_and(tid >= kRows || t0 + tid >= p.T || mine == 0);
  if (tid == 0) {
    s->n = n;
    s->uniform = n == 1 && all_first ? 1 : 0;
  }
  __syncthreads();
}

struct InnerCtl {
  uint64_t full[kInnerStages], empty[kInnerStages], done;
  uint32_t tmem_base;
  volatile int abort_flag;
  SlotList<kAM> slots;
  PairSlots pair;
  SlotScratch scratch;
  unsigned bad[kPairM / 32];
  float scale[kInnerCols / 16];   // of the group's slots
};

// Threads tid of n: part `part` of `parts` of the B of every adapter that a mixed block of 256 tokens names.
DEV void inner_look_through(const AdapterParams& p, InnerCtl& ctl, int part, int parts, int tid, int n) {
  if (ctl.pair.uniform || ctl.pair.n == 0) return;
  const size_t rows = p.swiglu_rows > 0 ? 2 * (size_t)p.M : (size_t)p.M;
  const size_t vec = rows * p.rank / 8, per = (vec + parts - 1) / parts;
  const size_t i0 = per * part < vec ? per * part : vec, i1 = i0 + per < vec ? i0 + per : vec;
  for (int s = 0; s < ctl.pair.n; ++s) {
    const uint4* B = reinterpret_cast<const uint4*>(p.B) + vec * ctl.pair.adapter[s];
    bool bad = false;
    for (size_t i = i0 + tid; i < i1; i += (size_t)n * 16) {   // sixteen loads in flight
      uint4 v[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = i + (size_t)k * n < i1 ? __ldg(B + i + (size_t)k * n) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int k = 0; k < 16; ++k) bad |= any_nonfinite(v[k]);
    }
    if (bad) atomicOr(&ctl.bad[s >> 5], 1u << (s & 31));
  }
}
DEV void inner_write_bad(const AdapterParams& p, const InnerCtl& ctl, int block, int part, int tid) {
  if (tid < kPairM / 32) p.bad[((size_t)block * kBadParts + part) * (kPairM / 32) + tid] = ctl.bad[tid];
}

__global__ void __launch_bounds__(kInnerThreads, 1)
adapter_inner_umma_kernel(const AdapterParams p, const __grid_constant__ CUtensorMap tm_x,
                          const __grid_constant__ CUtensorMap tm_a, const int r16) {
  cg::cluster_group cluster = cg::this_cluster();
  const int KS = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
  __shared__ InnerCtl ctl;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t0 = blockIdx.x * kAM, group = blockIdx.z;
  const int per_group = kInnerCols / r16;
  if (tid == 0) {   // set-up that touches no global memory: under the previous kernel's end
    for (int i = 0; i < kInnerStages; ++i) { mbar_init(&ctl.full[i], 1); mbar_init(&ctl.empty[i], 1); }
    mbar_init(&ctl.done, 1);
    ctl.abort_flag = 0;
    fence_barrier_init();
    prefetch_tensormap(&tm_x);
    prefetch_tensormap(&tm_a);
  }
  pdl_wait();                 // see adapter_inner_dot_kernel
  pdl_launch_dependents();
  build_slots<kAM>(p, t0, &ctl.slots, ctl.scratch, group == 0 && rank == 0);
  // the second launch's list, of this block and its neighbour; the slots whose B is not finite
  const int pair_block = blockIdx.x / 2, half = blockIdx.x & 1;
  if (group == 0) {
    build_slots<kPairM>(p, pair_block * kPairM, &ctl.pair, ctl.scratch, false);
    if (half == 0 && rank == KS - 1) {
      const int* src = reinterpret_cast<const int*>(&ctl.pair);
      int* dst = reinterpret_cast<int*>(p.slots + pair_block);
      for (int i = tid; i < (int)(sizeof(PairSlots) / 4); i += kInnerThreads) dst[i] = src[i];
    }
    if (tid < kPairM / 32) ctl.bad[tid] = 0u;
  }
  const int slot0 = group * per_group;
  const int cnt = min(ctl.slots.n - slot0, per_group);
  if (cnt <= 0) {             // the whole cluster
    if (group == 0) {
      __syncthreads();
      inner_look_through(p, ctl, half * KS + rank, (2 * pair_block + 1 < (int)gridDim.x ? 2 : 1) * KS, tid, kInnerThreads);
      __syncthreads();
      inner_write_bad(p, ctl, pair_block, half * KS + rank, tid);
    }
    return;
  }
  if (tid >= 64 && tid - 64 < cnt) ctl.scale[tid - 64] = __ldg(p.scale + ctl.slots.adapter[slot0 + tid - 64]);
  if (warp == 1) {
    tmem_alloc(&ctl.tmem_base, kInnerCols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = ctl.tmem_base;
  const int nkb_all = (p.K + kABK - 1) / kABK;
  const int nkb = (nkb_all - rank + KS - 1) / KS;
  volatile int* abort_flag = &ctl.abort_flag;

  if (warp == 0 && elect_one()) {
    const uint32_t bytes = (uint32_t)(kAXBytes + cnt * r16 * kABK * 2);
    int it = 0;
    for (; it < nkb; ++it) {
      const int s = it % kInnerStages;
      if (!mbar_wait_bounded(&ctl.empty[s], ((it / kInnerStages) & 1u) ^ 1u, abort_flag, p.dev_status, kWaitLimitClk)) break;
      const int k0 = (rank + it * KS) * kABK;
      unsigned char* st = ring + s * kInnerStageBytes;
      mbar_expect_tx(&ctl.full[s], bytes);
      tma_load_2d(st, &tm_x, &ctl.full[s], k0, t0);
      for (int i = 0; i < cnt; ++i)
        tma_load_3d(st + kAXBytes + i * r16 * 128, &tm_a, &ctl.full[s], k0, 0, ctl.slots.adapter[slot0 + i]);
    }
    for (int q = it > kInnerStages ? it - kInnerStages : 0; q < it; ++q)
      mbar_wait_drain(&ctl.full[q % kInnerStages], (q / kInnerStages) & 1u);
  } else if (warp == 1 && elect_one()) {
    const uint32_t idesc = umma_idesc_bf16(kAM, cnt * r16);
    for (int it = 0; it < nkb; ++it) {
      const int s = it % kInnerStages;
      if (!mbar_wait_bounded(&ctl.full[s], (it / kInnerStages) & 1u, abort_flag, p.dev_status, kWaitLimitClk)) break;
      tc_fence_after_sync();
      const uint32_t sa = smem_u32(ring + s * kInnerStageBytes);
      const uint64_t da = umma_desc_sw128(sa), db = umma_desc_sw128(sa + kAXBytes);
#pragma unroll
      for (int k = 0; k < kABK / 16; ++k)
        umma_bf16(tmem, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, (it | k) != 0 ? 1u : 0u);
      umma_commit(&ctl.empty[s]);
    }
    umma_commit(&ctl.done);
  } else if (warp >= 2 && group == 0) {
    inner_look_through(p, ctl, half * KS + rank, (2 * pair_block + 1 < (int)gridDim.x ? 2 : 1) * KS, tid - 64, kInnerThreads - 64);
  }
  __syncwarp();
  if (!mbar_spin_bounded_warp(&ctl.done, 0u, abort_flag, p.dev_status, 2 * kWaitLimitClk)) {
    ctl.abort_flag = 1;
    mbar_wait_drain(&ctl.done, 0u);
  }
  tc_fence_after_sync();
  __syncthreads();            // the ring is free: the partial inner values alias it
  if (group == 0) inner_write_bad(p, ctl, pair_block, half * KS + rank, tid);

  // every token's own columns: warp w reads TMEM lanes 32 (w % 4) .., its half of the 16-column steps
  const int RS = r16 + 1;
  float* part = reinterpret_cast<float*>(ring);
  const bool aborted = ctl.abort_flag != 0;
  {
    const int q = warp & 3, col_half = warp >> 2, row = q * 32 + lane;
    const int mine = ctl.slots.row_slot[row] - slot0;
    for (int i = 0; i < cnt; ++i) {
      if (__ballot_sync(0xffffffffu, mine == i) == 0u) continue;
      for (int c = col_half * 16; c < r16; c += 32) {
        uint32_t v[16];
        tmem_ld_32x16(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(i * r16 + c), v);
        tmem_ld_wait();
        if (mine == i) {
#pragma unroll
          for (int k = 0; k < 16; ++k) part[row * RS + c + k] = aborted ? __int_as_float(0x7fc00000) : __uint_as_float(v[k]);
        }
      }
    }
  }
  tc_fence_before_sync();
  cluster.sync();
  const float* peer[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) peer[k] = cluster.map_shared_rank(part, k < KS ? k : 0);
  const int nchunk = (p.rank + kRankChunk - 1) / kRankChunk, mine = kAM / KS / (kInnerThreads / 32) * nchunk;
#pragma unroll 4
  for (int i = 0; i < mine; ++i) {   // this warp's rows of the rank's share, a chunk a step, zeros behind the rank
    const int c = i % nchunk, row = rank + KS * (warp + kInnerThreads / 32 * (i / nchunk)), r = c * kRankChunk + lane;
    const int slot = ctl.slots.row_slot[row] - slot0;
    const bool used = slot >= 0 && slot < cnt;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = used && k < KS && r < p.rank ? peer[k][row * RS + r] : 0.f;
#pragma unroll
    for (int k = 1; k < 8; ++k) v[0] += v[k];
    if (!used) continue;
    const float f = r < p.rank ? ctl.scale[slot] * v[0] : 0.f;
    // a finite value that rounding would make infinite takes bf16's largest as its first term; the rest is below 2^121
    constexpr float kLargest = 3.3895313892515355e38f;
    const bool above = fabsf(f) > kLargest && fabsf(f) <= 3.402823466e38f;
    const __nv_bfloat16 hi = __float2bfloat16_rn(above ? copysignf(kLargest, f) : f);
    __nv_bfloat16* out = p.vt + ((size_t)(t0 + row) * nchunk + c) * (2 * kRankChunk) + lane;
    out[0] = hi;
    out[kRankChunk] = __float2bfloat16_rn(bf16_rest(f, __bfloat16_as_ushort(hi)));
  }
  cluster.sync();             // no CTA leaves while a peer reads its partial sums
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, kInnerCols);
  }
}

// ------------------------------------------------------------------------------------------------ the projection, few tokens
// Bound by streaming W, so the roles are turned round: a tile is 128 weight rows (UMMA M; with SwiGLU 64 rows of W1 and
// their 64 rows of W3) against all tokens (UMMA N = T rounded up to 16), and its K loop is split over a cluster of
// KS = 128 / kCols CTAs, which fills the SMs and keeps the number of stages each CTA has to issue small.  A stage costs its
// producer and its issuer the same whatever it holds, so it is two K blocks (`blocks`) where K allows it and W1's and W3's rows
// come in one load (13.4 -> 10.7 us at 64 tokens, K 2048, M 2816, with the inner values staged in shared memory).  The partial products pass through
// distributed shared memory; rank r adds them up, in rank order, for its kCols weight rows, adds the tokens' adapter terms
// and stores.  The adapter terms are summed on the CUDA cores while the loads are under way.
// With the inner values, from HBM: 1 token, K 2048, M 4096 6.8 us (2.5 TB/s of W); 64 tokens of 48 adapters, M 2816 10.5 us
// (1.8 TB/s of W and the adapters); both shared projections at 64 tokens (H 2048, S I 2816) 28.3 us (1.7 TB/s).  What is left
// above the bytes: two launches' set-up and drain, the exchange over the cluster, the tokens' B through few SMs.
constexpr int kFewThreads = 512;
constexpr int kFewTermWarps = kFewThreads / 32 - 2;
constexpr int kFewWBytes = 128 * kABK * 2;      // 16 KB
constexpr int kFewMaxStages = 8;

struct FewTile {
  int w_row, w_sub;       // first weight row (of W1) inside its sub-expert, the sub-expert
  int col0, col_limit;    // its output column; where the sub-expert's columns end
  size_t b_row;           // the same row in B's numbering
};

template <bool kGlu>
DEV FewTile few_tile(const AdapterParams& p, int tile) {
  FewTile t;
  if (kGlu) {
    const int per_sub = (p.swiglu_rows + 63) / 64;
    t.w_sub = tile / per_sub;
    t.w_row = (tile % per_sub) * 64;
    t.col0 = t.w_sub * p.swiglu_rows + t.w_row;
    t.col_limit = (t.w_sub + 1) * p.swiglu_rows;
    t.b_row = (size_t)t.w_sub * 2 * p.swiglu_rows + t.w_row;
  } else {
    t.w_sub = 0;
    t.w_row = t.col0 = tile * 128;
    t.col_limit = p.M;
    t.b_row = t.w_row;
  }
  return t;
}

// The adapter terms of this rank's weight rows, delta[token][kCols + 4]: lanes along the rows, so that what a token reads
// of its B is in one piece.  With SwiGLU the first half of the columns is W1's.  A warp takes every kFewTermWarps-th token
// (or pair of tokens, with 16 columns); a step is 16 ranks of kTok tokens, and the next step's B, which does not depend on
// the first launch, is on its way while the present one is summed -- the first step's already while that launch runs.
// Tokens without an adapter are left out.
template <int kCols, bool kGlu>
struct FewTerms {
  static constexpr int kWide = kCols < 32 ? kCols : 32, kPer = kCols / kWide, kSub = 32 / kWide, kTok = kPer >= 4 ? 1 : 4 / kPer;
  const AdapterParams& p;
  const int* ids;              // shared memory: the tokens' adapters
  float* vs;                   // shared memory: the inner values [T][rank]
  const uint16_t* Bc[kPer];
  bool col_ok[kPer];
  int first, c_lane, steps, per_group;
  size_t b_adapter;

  DEV FewTerms(const AdapterParams& p_, const FewTile& t, const int* ids_, float* vs_, int c_first, int w, int lane)
      : p(p_), ids(ids_), vs(vs_) {
    c_lane = lane % kWide;
    first = w * kSub + lane / kWide;
    b_adapter = (kGlu ? 2 * (size_t)p.M : (size_t)p.M) * p.rank;
    per_group = (p.rank + 15) / 16;
    const int stride = kFewTermWarps * kSub * kTok;   // tokens of all warps in one group
    steps = (p.T + stride - 1) / stride * per_group;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int c = c_lane + kWide * i;
      const bool up = kGlu && c >= kCols / 2;
      const int off = c_first + (up ? c - kCols / 2 : c);   // output column inside the tile
      col_ok[i] = t.col0 + off < t.col_limit;
      Bc[i] = p.B + (t.b_row + (col_ok[i] ? off + (up ? p.swiglu_rows : 0) : 0)) * p.rank;
    }
  }
  DEV int token(int step, int k) const { return first + ((step / per_group) * kTok + k) * kFewTermWarps * kSub; }
  DEV int adapter(int step, int k) const {
    const int t = token(step, k);
    return t < p.T ? ids[t] : -1;
  }
  DEV void load(int step, uint4 (&b)[kTok][kPer][2]) const {
    const int r = (step % per_group) * 16;
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      const int a = step < steps ? adapter(step, k) : -1;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          b[k][i][h] = make_uint4(0u, 0u, 0u, 0u);
          if (a >= 0 && r + 8 * h < p.rank) b[k][i][h] = __ldg(reinterpret_cast<const uint4*>(Bc[i] + a * b_adapter + r + 8 * h));
        }
    }
  }
  DEV void add(int step, const uint4 (&b)[kTok][kPer][2], float (&acc)[kTok][kPer], float* delta) const {
    const int r = (step % per_group) * 16;
    const bool last = step % per_group == per_group - 1;
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      if (adapter(step, k) >= 0) {
        const float4* v = reinterpret_cast<const float4*>(vs + token(step, k) * p.rank + r);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (r + 8 * h >= p.rank) continue;
          const float4 v0 = v[2 * h], v1 = v[2 * h + 1];
#pragma unroll
          for (int i = 0; i < kPer; ++i) acc[k][i] = fma8f(v0, v1, b[k][i][h], acc[k][i]);
        }
        if (last) {
#pragma unroll
          for (int i = 0; i < kPer; ++i)
            if (col_ok[i]) delta[token(step, k) * (kCols + 4) + c_lane + kWide * i] = acc[k][i];
        }
      }
      if (last) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) acc[k][i] = 0.f;
      }
    }
  }
  DEV void run(float* delta) const {
    uint4 b0[kTok][kPer][2], b1[kTok][kPer][2];
    float acc[kTok][kPer];
#pragma unroll
    for (int k = 0; k < kTok; ++k)
#pragma unroll
      for (int i = 0; i < kPer; ++i) acc[k][i] = 0.f;
    load(0, b0);
    pdl_wait();
    // the inner values of tokens without an adapter were not written; nothing uses them
    for (int i = threadIdx.x - 64; i < p.T * p.rank / 4; i += kFewTermWarps * 32)
      reinterpret_cast<float4*>(vs)[i] = __ldcg(reinterpret_cast<const float4*>(p.v) + i);
    asm volatile("bar.sync 1, %0;" ::"n"(kFewTermWarps * 32) : "memory");   // the warps that run this
    for (int s = 0; s < steps; s += 2) {
      load(s + 1, b1);
      add(s, b0, acc, delta);
      if (s + 1 < steps) {
        load(s + 2, b0);
        add(s + 1, b1, acc, delta);
      }
    }
  }
};

struct FewCtl {
  uint64_t full[kFewMaxStages], empty[kFewMaxStages], done;
  uint32_t tmem_base;
  volatile int abort_flag;
  int ids[kDotTokens];
};

// Place of weight row `row` of the tile in the partial product: the rank that finishes it, its column there.
template <int kCols, bool kGlu>
DEV int few_part_index(int row, int tokens, int token) {
  constexpr int kOuts = kGlu ? kCols / 2 : kCols;
  const int r = kGlu && row >= 64 ? row - 64 : row;
  const int col = r % kOuts + (kGlu && row >= 64 ? kOuts : 0);
  return ((r / kOuts) * tokens + token) * kCols + col;
}

template <int kCols, bool kGlu>
__global__ void __launch_bounds__(kFewThreads)
adapter_few_kernel(const AdapterParams p, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w,
                   const int t16, const int blocks, const int stages, const int ring_bytes) {
  constexpr int KS = 128 / kCols, kOuts = kGlu ? kCols / 2 : kCols;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = KS > 1 ? (int)cluster.block_rank() : 0;
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
  float* delta = reinterpret_cast<float*>(ring + ring_bytes);
  __shared__ FewCtl ctl;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int x_bytes = t16 * 128, stage_bytes = blocks * (kFewWBytes + x_bytes);   // W blocks, then x blocks
  const uint32_t tmem_cols = t16 <= 32 ? 32u : t16 <= 64 ? 64u : 128u;
  const FewTile t = few_tile<kGlu>(p, blockIdx.x);
  if (warp == 0) {
    if (lane < kFewMaxStages) { mbar_init(&ctl.full[lane], 1); mbar_init(&ctl.empty[lane], 1); }
    if (lane == kFewMaxStages) { mbar_init(&ctl.done, 1); ctl.abort_flag = 0; }
    fence_barrier_init();
    if (lane == 0) prefetch_tensormap(&tm_w);
    if (lane == 1) prefetch_tensormap(&tm_x);
  } else if (warp == 1) {
    tmem_alloc(&ctl.tmem_base, tmem_cols);
    tmem_relinquish();
  } else if (tid - 64 < p.T) {
    ctl.ids[tid - 64] = valid_adapter(__ldg(p.adapter_id + tid - 64), p.n_adapters);
  }
  pdl_launch_dependents();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = ctl.tmem_base;
  volatile int* abort_flag = &ctl.abort_flag;
  const int n_all = (p.K + kABK * blocks - 1) / (kABK * blocks), n_mine = (n_all - rank + KS - 1) / KS;   // rank, rank + KS, ...
  // x and W may be read at once, what the first launch writes after pdl_wait (see adapter_inner_dot_kernel)
  if (warp == 0) {
    if (elect_one()) {
      RingPos r;
      int it = 0;
      for (; it < n_mine; ++it, r.next(stages)) {
        if (!mbar_wait_bounded(&ctl.empty[r.s], r.ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk)) break;
        unsigned char* st = ring + r.s * stage_bytes;
        const int k0 = (rank + it * KS) * kABK * blocks;
        int sub = t.w_sub, kc = k0;
        if (!kGlu && p.k_per_sub > 0) { sub = k0 / p.k_per_sub; kc = k0 - sub * p.k_per_sub; }
        mbar_expect_tx(&ctl.full[r.s], (uint32_t)stage_bytes);
        if (blocks > 1) {
          tma_load_5d(st, &tm_w, &ctl.full[r.s], 0, t.w_row, 0, kc / kABK, sub);
          tma_load_5d(st + blocks * kFewWBytes, &tm_x, &ctl.full[r.s], 0, 0, 0, k0 / kABK, 0);
        } else {
          tma_load_5d(st, &tm_w, &ctl.full[r.s], kc, t.w_row, 0, 0, sub);
          tma_load_5d(st + kFewWBytes, &tm_x, &ctl.full[r.s], k0, 0, 0, 0, 0);
        }
      }
      for (int q = it > stages ? it - stages : 0; q < it; ++q) mbar_wait_drain(&ctl.full[q % stages], (q / stages) & 1u);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      const uint32_t idesc = umma_idesc_bf16(128, t16);
      RingPos r;
      for (int it = 0; it < n_mine; ++it, r.next(stages)) {
        if (!mbar_wait_bounded(&ctl.full[r.s], r.ph, abort_flag, p.dev_status, kWaitLimitClk)) break;
        tc_fence_after_sync();
        const uint32_t sw = smem_u32(ring + r.s * stage_bytes), sx = sw + blocks * kFewWBytes;
        for (int b = 0; b < blocks; ++b) {
          const uint64_t da = umma_desc_sw128(sw + b * kFewWBytes), db = umma_desc_sw128(sx + b * x_bytes);
#pragma unroll
          for (int k = 0; k < kABK / 16; ++k)
            umma_bf16(tmem, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, (it | b | k) != 0 ? 1u : 0u);
        }
        umma_commit(&ctl.empty[r.s]);
      }
      umma_commit(&ctl.done);
    }
  } else {
    FewTerms<kCols, kGlu>(p, t, ctl.ids, delta + p.T * (kCols + 4), rank * kOuts, warp - 2, lane).run(delta);
  }
  __syncwarp();
  if (lane == 0 && !mbar_wait_bounded(&ctl.done, 0u, abort_flag, p.dev_status, 2 * kWaitLimitClk)) mbar_wait_drain(&ctl.done, 0u);
  __syncwarp();
  tc_fence_after_sync();
  __syncthreads();            // loads landed, products complete: the partial product takes the ring's place
  float* part = reinterpret_cast<float*>(ring);
  if (warp < 4) {
    const int row = warp * 32 + lane;
    for (int c0 = 0; c0 < t16; c0 += 16) {
      uint32_t u[16];
      tmem_ld_32x16(tmem + ((uint32_t)(warp * 32) << 16) + (uint32_t)c0, u);
      tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < 16; ++i) part[few_part_index<kCols, kGlu>(row, t16, c0 + i)] = n_mine > 0 ? __uint_as_float(u[i]) : 0.f;
    }
  }
  tc_fence_before_sync();
  if (KS > 1) cluster.sync(); else __syncthreads();
  const float* peer[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) peer[k] = KS > 1 ? cluster.map_shared_rank(part, k) : part;
  pdl_wait();
  // eight output columns of one token a thread
  constexpr int kGroups = kOuts / 8;
  for (int i = tid; i < p.T * kGroups; i += kFewThreads) {
    const int row = i / kGroups, c = (i % kGroups) * 8, col = rank * kOuts + c;
    if (t.col0 + col >= t.col_limit) continue;
    float f[kGlu ? 16 : 8];
#pragma unroll
    for (int h = 0; h < (kGlu ? 4 : 2); ++h) {
      float4 v[KS];
#pragma unroll
      for (int k = 0; k < KS; ++k) v[k] = *reinterpret_cast<const float4*>(peer[k] + (rank * t16 + row) * kCols + (h >> 1) * kOuts + c + (h & 1) * 4);
#pragma unroll
      for (int k = 1; k < KS; ++k) { v[0].x += v[k].x; v[0].y += v[k].y; v[0].z += v[k].z; v[0].w += v[k].w; }
      f[4 * h] = v[0].x; f[4 * h + 1] = v[0].y; f[4 * h + 2] = v[0].z; f[4 * h + 3] = v[0].w;
    }
    if (ctl.ids[row] >= 0) {
      const float* d = delta + row * (kCols + 4) + c;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[e] += d[e];
        if constexpr (kGlu) f[8 + e] += d[kCols / 2 + e];
      }
    }
    if constexpr (kGlu) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = __fdividef(f[e], 1.f + __expf(-f[e])) * f[8 + e];
    }
    *reinterpret_cast<uint4*>(p.y + (size_t)row * p.M + t.col0 + col) =
        make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
  if (KS > 1) cluster.sync();   // no CTA leaves while a peer reads its partial product
  else __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, tmem_cols);
  }
}

// ------------------------------------------------------------------------------------------------ the projection, many tokens
// CTA pairs (tcgen05 cta_group::2): a tile is 256 tokens x nt weight rows (with SwiGLU nt/2 rows of W1 and their nt/2 rows of
// W3); each CTA of the pair loads its 128 tokens' x and half of the weight rows, so that a K block moves 16 KB + 64 nt bytes
// into each SM instead of 16 KB + 128 nt, which is what bounded one CTA a tile (600 clocks for 448 clocks of products at
// nt = 224; 64 us against 53 us at 4096 tokens).  Persistent over tiles, row blocks innermost so that concurrent pairs share
// a weight tile through L2; nt is chosen by adapter_pick_nt.  x and the weights have a producer each: at the adapter blocks
// they wait for different things.  With the inner values, from HBM: 4096 tokens, K 2048, M 2816, rank 64, 8 adapters in
// runs 56.3 us (0.88 PFLOP/s with the adapters' products, 0.64 of the sustained rate); both shared projections at 2045 tokens
// (H 2048, S I 2816, rank 32) 83.2 us (0.87 PFLOP/s).  The same product with no adapter named takes 39 us, with one adapter
// for all 49, with every token another of the eight 100: the inner values come before the first tile's end, and every adapter
// of a block adds two K blocks to its tiles.  200 tokens, each of another request, 64 adapters of rank 16: 110 us, 64 K blocks
// behind the 32 of K on 36 SMs.
// In each CTA: warp 0 W and B loads; warp 1 (leader) MMA issuer; warps 2-9 epilogue; 10-17 the masked V tiles of mixed
// blocks, two groups of four in turn; 18 x loads, and V's where a block names one adapter.  Two accumulators in TMEM: a
// tile's epilogue (TMEM -> registers -> shared memory -> TMA store) runs under the next tile's K loop.
// The masked V of both CTAs is an operand of the leader's products, so the peer's V warps release it at cluster scope, each
// for itself, and the issuer acquires it there: 3 us of the 56 and 15 of the 100 above.  A warp that gathers a CTA's four
// arrivals and passes them on was slower (60 and 108 us): a cluster-scope release takes longer than a K block.
constexpr int kAdThreads = 608;
constexpr int kAdSmem = 226 * 1024;
constexpr int kAdMaxStages = 8;
constexpr int kAdOutBytes = 8 * 4096; // per epilogue warp two buffers of 32 rows x 32 columns

struct AdCtl {
  uint64_t full[kAdMaxStages];      // leader's: the stage's loads have landed in both CTAs
  uint64_t empty[kAdMaxStages];     // the stage's products are complete
  uint64_t vstart[2][kAdMaxStages]; // the stage is free for masked V, of the one or the other group of V warps
  uint64_t vfull[kAdMaxStages];     // leader's: masked V is written in both CTAs
  uint64_t tmem_full[2], tmem_empty[2], drain;
  uint32_t tmem_base;
  volatile uint32_t progress;       // K blocks whose x (or V) the CTA has asked for
  volatile int abort_flag;
};

struct AdTile {
  int block, m0;
  int row, sub;          // first row of the (W1) weight tile inside its sub-expert = first output column there
  int rows_left;         // output columns of the sub-expert from there on
};

template <bool kGlu>
DEV AdTile ad_tile(const AdapterParams& p, int tile, int mblocks, int nt) {
  const int out = kGlu ? nt / 2 : nt, nb = tile / mblocks;
  AdTile t;
  t.block = tile - nb * mblocks;
  t.m0 = t.block * kPairM;
  const int rows = kGlu ? p.swiglu_rows : p.M, per_sub = (rows + out - 1) / out;
  t.sub = nb / per_sub;
  t.row = (nb - t.sub * per_sub) * out;
  t.rows_left = rows - t.row;
  return t;
}

// Slots 32 w .. of a mixed block whose B is not finite.
DEV unsigned bad_slots(const AdapterParams& p, int block, int mblocks128, int w) {
  const int parts = (2 * block + 1 < mblocks128 ? 2 : 1) * p.parts;
  const unsigned* b = p.bad + (size_t)block * kBadParts * (kPairM / 32) + w;
  unsigned v = 0u;
#pragma unroll
  for (int i = 0; i < kBadParts; ++i)
    if (i < parts) v |= __ldcg(b + i * (kPairM / 32));
  return v;
}

// acc[i] += the row's adapter term, sum over the ranks of v[r] B[row + i][r], one token a lane (rare: B was not finite).
template <int kC>
DEV void add_adapter_term(const AdapterParams& p, const __nv_bfloat16* vt, const uint16_t* B, int rows_left, uint32_t (&acc)[kC]) {
#pragma unroll
  for (int i = 0; i < kC; ++i) {
    if (i >= rows_left) break;
    float sum = __uint_as_float(acc[i]);
#pragma unroll 1
    for (int r = 0; r < p.rank; ++r) {
      const __nv_bfloat16* v = vt + (r / kRankChunk) * (2 * kRankChunk) + r % kRankChunk;
      sum = fmaf(__bfloat162float(v[0]) + __bfloat162float(v[kRankChunk]), bf16_bits_to_float((uint32_t)B[(size_t)i * p.rank + r]), sum);
    }
    acc[i] = __float_as_uint(sum);
  }
}

template <bool kGlu>
__global__ void __launch_bounds__(kAdThreads, 1)
adapter_linear_kernel(const AdapterParams p, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w,
                      const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_v,
                      const __grid_constant__ CUtensorMap tm_y, const int nt, const int stages, const int mblocks,
                      const int total_tiles) {
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
  const int w_bytes = nt * kABK, stage_bytes = kAXBytes + w_bytes, out_cols = kGlu ? nt / 2 : nt;   // w_bytes: half the tile's rows
  unsigned char* out_tiles = ring + stages * stage_bytes;
  __shared__ AdCtl ctl;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster_cta_rank();          // 0 = leader
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  if (warp == 0) {
    if (lane < kAdMaxStages) {
      mbar_init(&ctl.full[lane], 4);
      mbar_init(&ctl.empty[lane], 1);
      mbar_init(&ctl.vstart[0][lane], 1);
      mbar_init(&ctl.vstart[1][lane], 1);
      mbar_init(&ctl.vfull[lane], 8);
    } else if (lane < kAdMaxStages + 2) {
      mbar_init(&ctl.tmem_full[lane - kAdMaxStages], 1);
      mbar_init(&ctl.tmem_empty[lane - kAdMaxStages], 16);
    } else if (lane == kAdMaxStages + 2) {
      mbar_init(&ctl.drain, 1);
      ctl.progress = 0u;
      ctl.abort_flag = 0;
    }
    fence_barrier_init();
    if (lane == 0) prefetch_tensormap(&tm_x);
    if (lane == 1) prefetch_tensormap(&tm_w);
    if (lane == 2) prefetch_tensormap(&tm_b);
    if (lane == 3) prefetch_tensormap(&tm_y);
    if (lane == 4) prefetch_tensormap(&tm_v);
  } else if (warp == 1) {
    tmem_alloc_pair(&ctl.tmem_base, 512);
    tmem_relinquish_pair();
  }
  pdl_launch_dependents();
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync_all();          // both CTAs' barriers are initialised before either signals the other
  tc_fence_after_sync();
  const uint32_t tmem_base = ctl.tmem_base;
  volatile int* abort_flag = &ctl.abort_flag;
  // The first launch lets this one start once everything before it is complete: x and W may be read at once, its own
  // results (vt, slots, bad) after pdl_wait.
  const int nkb = (p.K + kABK - 1) / kABK;
  const int k_sub = p.k_per_sub > 0 ? p.k_per_sub : nkb * kABK;   // K per sub-expert of W
  const int nchunk = (p.rank + kRankChunk - 1) / kRankChunk, mblocks128 = (p.T + kAM - 1) / kAM;
  auto slots_of = [&](int block) { return min(__ldcg(&p.slots[block].n), kPairM); };

  if (warp == 0) {
    // ======================= W and B loads =======================
    if (elect_one()) {
      RingPos r;
      uint32_t issued = 0;
      bool ok = true;
      const int w_row = kGlu ? 0 : rank * (nt / 2), w_half = kGlu ? rank : 0;   // this CTA's half of a tile's weight rows
      for (int tile = pair; ok && tile < total_tiles; tile += n_pairs) {
        const AdTile t = ad_tile<kGlu>(p, tile, mblocks, nt);
        const bool first = tile == pair;
        const PairSlots* sl = p.slots + t.block;
        int n_slots = first ? 0 : slots_of(t.block), next = first ? 0 : __ldcg(&sl->adapter[0]);
        int sub = kGlu ? t.sub : 0, kc = 0;
        for (int kb = 0; kb < nkb; ++kb, r.next(stages), ++issued) {
          if (!(ok = mbar_wait_bounded(&ctl.empty[r.s], r.ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
          const uint32_t bar = cluster_addr_of(&ctl.full[r.s], 0);
          mbar_expect_tx_cluster(bar, (uint32_t)w_bytes);
          tma_load_5d_pair(ring + r.s * stage_bytes + kAXBytes, &tm_w, bar, kc, t.row + w_row, w_half, 0, sub);
          kc += kABK;
          if (!kGlu && kc >= k_sub) { kc = 0; ++sub; }
        }
        if (!ok) break;
        if (first) {
          pdl_wait();
          n_slots = slots_of(t.block);
          next = __ldcg(&sl->adapter[0]);
        }
        for (int i = 0; ok && i < n_slots; ++i) {
          const int a = min(max(next, 0), p.n_adapters - 1);
          next = __ldcg(&sl->adapter[min(i + 1, kPairM - 1)]);
          for (int c = 0; c < nchunk; ++c, r.next(stages), ++issued) {
            if (!(ok = mbar_wait_bounded(&ctl.empty[r.s], r.ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
            const uint32_t bar = cluster_addr_of(&ctl.full[r.s], 0);
            mbar_expect_tx_cluster(bar, (uint32_t)w_bytes);
            tma_load_5d_pair(ring + r.s * stage_bytes + kAXBytes, &tm_b, bar, c * kRankChunk, t.row + w_row, w_half,
                             kGlu ? t.sub : 0, a);
          }
        }
      }
      // every load has landed before the CTA may exit: its products are complete
      for (uint32_t q = issued > (uint32_t)stages ? issued - stages : 0u; q < issued; ++q)
        mbar_wait_drain(&ctl.empty[q % stages], (q / stages) & 1u);
    }
  } else if (warp == 18) {
    // ======================= x loads, V loads of blocks with one adapter =======================
    if (elect_one()) {
      RingPos r;
      uint32_t issued = 0, turn = 0;
      bool ok = true;
      for (int tile = pair; ok && tile < total_tiles; tile += n_pairs) {
        const int block = tile % mblocks;
        const bool first = tile == pair;
        int n_slots = first ? 0 : slots_of(block), uniform = first ? 0 : __ldcg(&p.slots[block].uniform);
        for (int kb = 0; kb < nkb; ++kb, r.next(stages), ++issued) {
          if (!(ok = mbar_wait_bounded(&ctl.empty[r.s], r.ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
          const uint32_t bar = cluster_addr_of(&ctl.full[r.s], 0);
          mbar_expect_tx_cluster(bar, (uint32_t)kAXBytes);
          tma_load_2d_pair(ring + r.s * stage_bytes, &tm_x, bar, kb * kABK, block * kPairM + rank * kAM);
          ctl.progress = issued;
        }
        if (!ok) break;
        if (first) {
          pdl_wait();
          n_slots = slots_of(block);
          uniform = __ldcg(&p.slots[block].uniform);
        }
        for (int i = 0; i < n_slots * nchunk; ++i, r.next(stages), ++issued) {
          if (!(ok = mbar_wait_bounded(&ctl.empty[r.s], r.ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
          const uint32_t bar = cluster_addr_of(&ctl.full[r.s], 0);
          if (uniform) {
            mbar_expect_tx_cluster(bar, (uint32_t)kAXBytes);
            tma_load_2d_pair(ring + r.s * stage_bytes, &tm_v, bar, i * 2 * kRankChunk, block * kPairM + rank * kAM);
          } else {
            mbar_arrive(&ctl.vstart[turn][r.s]);   // the stage's V is a group of V warps'
            turn ^= 1u;
            mbar_arrive_cluster(bar);
          }
          ctl.progress = issued;
        }
      }
      for (uint32_t q = issued > (uint32_t)stages ? issued - stages : 0u; q < issued; ++q)
        mbar_wait_drain(&ctl.empty[q % stages], (q / stages) & 1u);
    }
  } else if (warp == 1) {
    // ======================= MMA issuer (leader) =======================
    if (rank == 0 && elect_one()) {
      const uint32_t idesc = umma_idesc_bf16(kPairM, nt);
      RingPos r;
      uint32_t tcount = 0, vphase = 0;
      bool ok = true;
      for (int tile = pair; ok && tile < total_tiles; tile += n_pairs, ++tcount) {
        const uint32_t a = tcount & 1u;
        const int block = tile % mblocks;
        const bool first = tile == pair;
        int n_slots = 0, uniform = 1;
        unsigned bad = 0u, words[kBadParts];
        // the loads of a later tile's list are under way during its K loop: nothing of them is used before its end
        const int parts = (2 * block + 1 < mblocks128 ? 2 : 1) * p.parts;
        auto look = [&]() {
          n_slots = __ldcg(&p.slots[block].n);
          uniform = __ldcg(&p.slots[block].uniform);
#pragma unroll
          for (int i = 0; i < kBadParts; ++i) words[i] = __ldcg(p.bad + ((size_t)block * kBadParts + min(i, parts - 1)) * (kPairM / 32));
        };
        if (!first) look();
        if (!(ok = mbar_wait_bounded(&ctl.tmem_empty[a], ((tcount >> 1) & 1u) ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
        tc_fence_after_sync();
        const uint32_t d = tmem_base + a * 256;
        for (int kb = 0; kb < nkb; ++kb, r.next(stages)) {
          if (!(ok = mbar_wait_bounded(&ctl.full[r.s], r.ph, abort_flag, p.dev_status, kWaitLimitClk))) break;
          tc_fence_after_sync();
          const uint32_t sa = smem_u32(ring + r.s * stage_bytes);
          const uint64_t da = umma_desc_sw128(sa), db = umma_desc_sw128(sa + kAXBytes);
#pragma unroll
          for (int k = 0; k < kABK / 16; ++k)
            umma_bf16_pair(d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, (kb | k) != 0 ? 1u : 0u);
          umma_commit_pair(&ctl.empty[r.s], 3);      // frees the stage in both CTAs
        }
        if (ok) {
          if (first) {
            pdl_wait();
            look();
          }
          n_slots = min(n_slots, kPairM);
#pragma unroll
          for (int i = 0; i < kBadParts; ++i) bad |= uniform ? 0u : words[i];
          for (int i = 0; ok && i < n_slots; ++i) {
            if (!uniform && i > 0 && (i & 31) == 0) bad = bad_slots(p, block, mblocks128, i >> 5);
            for (int c = 0; c < nchunk; ++c, r.next(stages)) {
              const int s = r.s;
              if (!uniform) {
                // V of the peer CTA's rows was written by its threads
                if (!(ok = mbar_wait_acquire_cluster(&ctl.vfull[s], (vphase >> s) & 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
                vphase ^= 1u << s;
              }
              if (!(ok = mbar_wait_bounded(&ctl.full[s], r.ph, abort_flag, p.dev_status, kWaitLimitClk))) break;
              tc_fence_after_sync();
              if (!((bad >> (i & 31)) & 1u)) {       // else the epilogue adds the slot's terms
                const uint32_t sa = smem_u32(ring + s * stage_bytes);
                const uint64_t da = umma_desc_sw128(sa), db = umma_desc_sw128(sa + kAXBytes);
                const int ranks = min(p.rank - c * kRankChunk, kRankChunk);
                for (int k = 0; k * 16 < ranks; ++k) {
                  umma_bf16_pair(d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, 1u);         // hi
                  umma_bf16_pair(d, da + (uint64_t)(k * 2 + 4), db + (uint64_t)(k * 2), idesc, 1u);     // lo
                }
              }
              umma_commit_pair(&ctl.empty[s], 3);
            }
          }
        }
        if (ok) umma_commit_pair(&ctl.tmem_full[a], 3);
      }
      umma_commit_pair(&ctl.drain, 1);
      mbar_wait_drain(&ctl.drain, 0u);
    }
  } else if (warp < 10) {
    // ======================= epilogue: two warps per quarter of the rows, every other 32 columns =======================
    const int q = warp & 3, half = (warp - 2) >> 2;
    unsigned char* mine = out_tiles + (warp - 2) * 4096;
    uint32_t tcount = 0, stores = 0;
    bool ok = true;
    const size_t b_rows = kGlu ? 2 * (size_t)p.M : (size_t)p.M;
    const int sub_rows = kGlu ? p.swiglu_rows : p.M;
    for (int tile = pair; ok && tile < total_tiles; tile += n_pairs, ++tcount) {
      const AdTile t = ad_tile<kGlu>(p, tile, mblocks, nt);
      const uint32_t a = tcount & 1u;
      if (tcount == 0) pdl_wait();
      const int row0 = t.m0 + rank * kAM + q * 32, row = row0 + lane;
      const bool row_ok = row < p.T;
      // the adapter whose term is still missing in this row
      int ad = -1;
      if (row_ok && __ldcg(&p.slots[t.block].uniform) == 0) {
        const int slot = __ldcg(&p.slots[t.block].row_slot[row - t.m0]);
        if (slot >= 0 && slot < kPairM && ((bad_slots(p, t.block, mblocks128, slot >> 5) >> (slot & 31)) & 1u))
          ad = min(max(__ldcg(&p.slots[t.block].adapter[slot]), 0), p.n_adapters - 1);
      }
      const bool any_ad = __any_sync(0xffffffffu, ad >= 0);
      if (!(ok = mbar_spin_progress_warp(&ctl.tmem_full[a], (tcount >> 1) & 1u, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk))) break;
      tc_fence_after_sync();
      const __nv_bfloat16* vt = p.vt + (size_t)(row_ok ? row : 0) * nchunk * (2 * kRankChunk);
      const size_t b_row = (size_t)t.sub * (kGlu ? 2 * sub_rows : sub_rows) + t.row;
      const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + a * 256;
      if (row0 < p.T) {
        constexpr int kC = kGlu ? 16 : 32;
        const int cols = min(out_cols, t.rows_left);
#pragma unroll 1
        for (int c0 = half * 32; c0 < cols; c0 += (kGlu && (c0 & 16) == 0) ? 16 : kGlu ? 48 : 64) {
          uint32_t u[kC];
          if constexpr (kGlu) {
            uint32_t g[kC];
            tmem_ld_32x16(taddr + (uint32_t)c0, u);
            tmem_ld_32x16(taddr + (uint32_t)(out_cols + c0), g);
            tmem_ld_wait();
            if (any_ad) {
              if (ad >= 0) {
                const uint16_t* Bt = p.B + ((size_t)ad * b_rows + b_row + c0) * p.rank;
                add_adapter_term<kC>(p, vt, Bt, t.rows_left - c0, u);
                add_adapter_term<kC>(p, vt, Bt + (size_t)sub_rows * p.rank, t.rows_left - c0, g);
              }
              __syncwarp();
            }
#pragma unroll
            for (int i = 0; i < kC; ++i) {
              const float z = __uint_as_float(u[i]);
              u[i] = __float_as_uint(__fdividef(z, 1.f + __expf(-z)) * __uint_as_float(g[i]));
            }
          } else {
            tmem_ld_32x32(taddr + (uint32_t)c0, u);
            tmem_ld_wait();
            if (any_ad) {
              if (ad >= 0) add_adapter_term<kC>(p, vt, p.B + ((size_t)ad * b_rows + b_row + c0) * p.rank, t.rows_left - c0, u);
              __syncwarp();
            }
          }
          // 32 columns a store: with SwiGLU two steps share a buffer
          const int col = kGlu ? c0 & 31 : 0;
          unsigned char* buf = mine + (stores & 1u) * 2048;
          if (col == 0) {
            if (lane == 0) bulk_wait_read<1>();   // the store before the last has read its buffer
            __syncwarp();
          }
#pragma unroll
          for (int i = 0; i < kC; i += 8)
            *reinterpret_cast<uint4*>(buf + lane * 64 + ((((col + i) / 8) ^ ((lane >> 1) & 3)) << 4)) =
                make_uint4(pack_bf16x2(__uint_as_float(u[i]), __uint_as_float(u[i + 1])),
                           pack_bf16x2(__uint_as_float(u[i + 2]), __uint_as_float(u[i + 3])),
                           pack_bf16x2(__uint_as_float(u[i + 4]), __uint_as_float(u[i + 5])),
                           pack_bf16x2(__uint_as_float(u[i + 6]), __uint_as_float(u[i + 7])));
          if (col + kC == 32) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              tma_store_5d(buf, &tm_y, t.row + c0 + kC - 32, t.sub, row0, 0, 0);
              bulk_commit();
            }
            ++stores;
          } else if (kGlu && c0 + kC >= cols && row_ok) {   // a last half of a buffer goes by plain stores
            uint4* out = reinterpret_cast<uint4*>(p.y + (size_t)row * p.M + (size_t)t.sub * sub_rows + t.row + c0);
#pragma unroll
            for (int i = 0; i < kC; i += 8)
              if (c0 + i < cols) out[i / 8] = *reinterpret_cast<const uint4*>(buf + lane * 64 + ((((col + i) / 8) ^ ((lane >> 1) & 3)) << 4));
          }
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(cluster_addr_of(&ctl.tmem_empty[a], 0));
    }
    if (lane == 0) bulk_wait_all();
  } else {
    // ======================= masked V of mixed blocks (warps 10-13 and 14-17, every other K block) =======================
    const int row = ((warp - 10) & 3) * 32 + lane, turn = (warp - 10) >> 2;
    RingPos r;
    uint32_t vphase = 0, count = 0;
    bool ok = true;
    pdl_wait();
    for (int tile = pair; ok && tile < total_tiles; tile += n_pairs) {
      const int block = tile % mblocks;
      const PairSlots* sl = p.slots + block;
      const int n_slots = slots_of(block), mine = __ldcg(&sl->row_slot[rank * kAM + row]);
      r.skip(nkb, stages);
      if (__ldcg(&sl->uniform)) {
        r.skip(n_slots * nchunk, stages);
        continue;
      }
      const uint4* v = reinterpret_cast<const uint4*>(p.vt + (size_t)(block * kPairM + rank * kAM + row) * nchunk * (2 * kRankChunk));
      uint4 f[8];   // the row's next chunk of inner values for this group
      auto fetch = [&](int c) {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = c < nchunk ? __ldcg(v + c * 8 + k) : make_uint4(0u, 0u, 0u, 0u);
      };
      // the row's chunks are those of K blocks mine * nchunk + c: the first of this group's, then every other one
      if (mine >= 0) fetch(((count + (uint32_t)(mine * nchunk)) & 1u) == (uint32_t)turn ? 0 : 1);
      for (int i = 0; ok && i < n_slots; ++i) {
        for (int c = 0; c < nchunk; ++c, ++count, r.next(stages)) {
          const int s = r.s;
          if ((count & 1u) != (uint32_t)turn) continue;
          // the x producer announces the stage: these warps do not follow the K loop's phases of empty[s].  Each group has
          // its own barriers: of another's it could fall two phases behind
          ok = mbar_spin_progress_warp(&ctl.vstart[turn][s], (vphase >> s) & 1u, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk);
          if (!ok) break;
          vphase ^= 1u << s;
          unsigned char* sa = ring + s * stage_bytes + row * 128;
          const bool own = mine == i;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            *reinterpret_cast<uint4*>(sa + ((k ^ (row & 7)) << 4)) = own ? f[k] : make_uint4(0u, 0u, 0u, 0u);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (rank == 0) mbar_arrive(&ctl.vfull[s]);
            else mbar_arrive_release_cluster(cluster_addr_of(&ctl.vfull[s], 0));   // the leader's product reads it
          }
          if (own) fetch(c + 2);
        }
      }
    }
  }
  pdl_wait();   // also where no role came to it: this launch ends after the one before it
  // neither CTA leaves, or frees TMEM, while its peer may still touch it
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

}  // namespace allocmoe

using namespace allocmoe;

namespace {

size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
// CTAs of a cluster: the largest power of two up to 8 and `most` that leaves about a CTA per SM for `clusters` of them.  An
// SM holds one such CTA, and 15 clusters of eight are resident at a time (33 of four): a sixteenth would wait for a second
// round (measured 15 us against 8 us for the inner values of 16 blocks).
int cluster_size(long long clusters, int most, int sms) {
  int n = 1;
  while (n < 8 && n * 2 <= most && clusters * n * 2 <= (n == 4 ? 15 * 8 : sms)) n *= 2;
  return n;
}
int token_blocks(int T) { return (T + kAM - 1) / kAM; }
int pair_blocks(int T) { return (T + kPairM - 1) / kPairM; }
size_t vt_bytes(int T, int rank) { return align256((size_t)T * ((rank + kRankChunk - 1) / kRankChunk) * 2 * kRankChunk * 2); }

int sm_count() {
  static PerDeviceInt cache;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  int n = cache.get(dev);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    cache.set(dev, n);
  }
  return n;
}

// Weight rows per tile: what makes rounds of tiles x time per tile smallest.  Measured clocks per K block: 340 for nt up to
// 192, 400 at 224, 460 at 256 -- so nothing below 160 can win.
int adapter_pick_nt(const AdapterArgs& a, int sms) {
  const bool glu = a.swiglu_rows > 0;
  int best = 0;
  double best_cost = 0;
  for (int nt = 256; nt >= 160; nt -= 32) {
    const int out = glu ? nt / 2 : nt, rows = glu ? a.swiglu_rows : a.M;
    const long long tiles = (long long)(a.M / rows) * ((rows + out - 1) / out) * pair_blocks(a.T);
    const double cost = (double)((tiles + sms / 2 - 1) / (sms / 2)) * (nt > 190 ? nt : 190);
    if (best == 0 || cost < best_cost) { best = nt; best_cost = cost; }
  }
  return best;
}

// x as (K, tokens, 1, blocks of K, 1): with blocked, K in blocks of 64 (coordinates (0, token, 0, block, 0)), else whole
// ((column, token, 0, 0, 0)).
Tensor5 input_tensor(const AdapterArgs& a, bool blocked) {
  Tensor5 t;
  const uint64_t K = (uint64_t)a.K;
  t.dim[0] = blocked ? 64 : K;
  t.dim[1] = (uint64_t)a.T;
  t.dim[3] = blocked ? K / 64 : 1;
  t.stride[0] = t.stride[1] = K;
  t.stride[2] = blocked ? 64 : K;
  return t;
}

// W as (K, rows, W1 and W3, blocks of K, sub-experts), K blocked in the same way.
Tensor5 weight_tensor(const AdapterArgs& a, bool blocked) {
  Tensor5 t;
  const bool glu = a.swiglu_rows > 0;
  const uint64_t K = a.k_per_sub > 0 ? (uint64_t)a.k_per_sub : (uint64_t)a.K;
  const uint64_t rows = glu ? (uint64_t)a.swiglu_rows : (uint64_t)a.M;
  t.dim[0] = blocked ? 64 : K;
  t.dim[1] = rows;
  t.dim[2] = glu ? 2 : 1;
  t.dim[3] = blocked ? K / 64 : 1;
  t.dim[4] = glu ? (uint64_t)(a.M / a.swiglu_rows) : (uint64_t)a.K / K;
  t.stride[0] = K;
  t.stride[1] = rows * K;
  t.stride[2] = blocked ? 64 : K;
  t.stride[3] = t.dim[2] * rows * K;
  return t;
}

// B as (rank, rows, W1's and W3's, sub-experts, adapters).
Tensor5 b_tensor(const AdapterArgs& a) {
  Tensor5 t;
  const bool glu = a.swiglu_rows > 0;
  const uint64_t r = (uint64_t)a.rank, rows = glu ? (uint64_t)a.swiglu_rows : (uint64_t)a.M;
  t.dim[0] = r;
  t.dim[1] = rows;
  t.dim[2] = glu ? 2 : 1;
  t.dim[3] = glu ? (uint64_t)(a.M / a.swiglu_rows) : 1;
  t.dim[4] = (uint64_t)a.n_adapters;
  t.stride[0] = r;
  t.stride[1] = rows * r;
  t.stride[2] = t.dim[2] * rows * r;
  t.stride[3] = t.dim[3] * t.stride[2];
  return t;
}

// y as (columns of a sub-expert, sub-experts, tokens, 1, 1).
Tensor5 output_tensor(const AdapterArgs& a) {
  Tensor5 t;
  const bool glu = a.swiglu_rows > 0;
  t.dim[0] = glu ? (uint64_t)a.swiglu_rows : (uint64_t)a.M;
  t.dim[1] = glu ? (uint64_t)(a.M / a.swiglu_rows) : 1;
  t.dim[2] = (uint64_t)a.T;
  t.stride[0] = t.dim[0];
  t.stride[1] = t.stride[2] = t.stride[3] = (uint64_t)a.M;
  return t;
}

template <bool kGlu>
moe_status launch_many(const AdapterArgs& a, const AdapterParams& p, int sms) {
  const int nt = adapter_pick_nt(a, sms), out = kGlu ? nt / 2 : nt;
  const int stage = kAXBytes + nt * kABK;
  const int stages = (kAdSmem - kAdOutBytes - 1024) / stage;   // 6 or 7
  const size_t smem = (size_t)stages * stage + kAdOutBytes + 1024;
  CUtensorMap tm_x, tm_w, tm_b, tm_v, tm_y;
  const uint64_t v_cols = (uint64_t)((a.rank + kRankChunk - 1) / kRankChunk) * 2 * kRankChunk;
  const uint32_t box_w[5] = {64, (uint32_t)nt / 2, 1, 1, 1}, box_y[5] = {32, 1, 32, 1, 1};
  if (!make_tmap(&tm_x, a.x, (uint64_t)a.K, (uint64_t)a.T, 0, (uint64_t)a.K, 0, kAM) ||
      !make_tmap5(&tm_w, a.W, weight_tensor(a, false), box_w, 128) || !make_tmap5(&tm_b, a.B, b_tensor(a), box_w, 128) ||
      !make_tmap(&tm_v, p.vt, v_cols, (uint64_t)a.T, 0, v_cols, 0, kAM) || !make_tmap5(&tm_y, a.y, output_tensor(a), box_y, 64))
    return MOE_ERR_CUDA;
  static PerDeviceOnce attr_set;
  if (!ensure_dynamic_smem(adapter_linear_kernel<kGlu>, kAdSmem, attr_set)) return MOE_ERR_CUDA;
  const int rows = kGlu ? a.swiglu_rows : a.M, mblocks = pair_blocks(a.T);
  const long long tiles = (long long)(a.M / rows) * ((rows + out - 1) / out) * mblocks;
  if (tiles >= (1ll << 31) - 4096) return MOE_ERR_ARG;
  const unsigned grid = 2u * (unsigned)(tiles < sms / 2 ? tiles : sms / 2);
  return launch_dependent_cluster(adapter_linear_kernel<kGlu>, dim3(grid), dim3(kAdThreads), smem, a.stream, dim3(2, 1, 1), p, tm_x,
                                  tm_w, tm_b, tm_v, tm_y, nt, stages, mblocks, (int)tiles) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}

template <int kCols, bool kGlu>
moe_status launch_few_t(const AdapterArgs& a, const AdapterParams& p, int tiles) {
  constexpr unsigned KS = 128 / kCols;
  CUtensorMap tm_x, tm_w;
  const int t16 = (a.T + 15) / 16 * 16;
  // two K blocks a stage where that divides K (a sub-expert's, too) and leaves every CTA of the cluster one
  const uint64_t kw = a.k_per_sub > 0 ? (uint64_t)a.k_per_sub : (uint64_t)a.K;
  const int blocks = kw % 128 == 0 && a.K >= 128 * (int)KS && a.T * (kCols + a.rank) <= 16384 ? 2 : 1;
  const Tensor5 x = input_tensor(a, blocks > 1), w = weight_tensor(a, blocks > 1);
  const uint32_t box_x[5] = {64, (uint32_t)t16, 1, (uint32_t)blocks, 1};
  const uint32_t box_w[5] = {64, kGlu ? 64u : 128u, kGlu ? 2u : 1u, (uint32_t)blocks, 1};
  if (!make_tmap5(&tm_x, a.x, x, box_x, 128) || !make_tmap5(&tm_w, a.W, w, box_w, 128)) return MOE_ERR_CUDA;
  const int stage = blocks * (kFewWBytes + t16 * 128), delta = a.T * (kCols + 4 + a.rank) * 4;   // and the inner values
  const int n = ((a.K + kABK * blocks - 1) / (kABK * blocks) + (int)KS - 1) / (int)KS;
  int stages = (216 * 1024 - delta) / stage;        // two at least: 128 tokens of rank 128, one CTA a tile
  if (stages > n) stages = n;
  if (stages > kFewMaxStages) stages = kFewMaxStages;
  int ring = stages * stage;
  const int part = t16 * 128 * 4;
  if (ring < part) ring = (part + 1023) / 1024 * 1024;
  const size_t smem = (size_t)ring + delta + 1024;
  static PerDeviceOnce attr_set;
  if (!ensure_dynamic_smem(adapter_few_kernel<kCols, kGlu>, 224 * 1024, attr_set)) return MOE_ERR_CUDA;
  return launch_dependent(adapter_few_kernel<kCols, kGlu>, dim3((unsigned)tiles, KS), dim3(kFewThreads), smem, a.stream, KS, p, tm_x,
                          tm_w, t16, blocks, stages, ring) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}

template <bool kGlu>
moe_status launch_few(const AdapterArgs& a, const AdapterParams& p, int sms) {
  const long long tiles = kGlu ? (long long)(a.M / a.swiglu_rows) * ((a.swiglu_rows + 63) / 64) : (a.M + 127) / 128;
  if (tiles >= (1ll << 31) / 8) return MOE_ERR_ARG;
  switch (cluster_size(tiles, (a.K + kABK - 1) / kABK, sms)) {
    case 1: return launch_few_t<128, kGlu>(a, p, (int)tiles);
    case 2: return launch_few_t<64, kGlu>(a, p, (int)tiles);
    case 4: return launch_few_t<32, kGlu>(a, p, (int)tiles);
    default: return launch_few_t<16, kGlu>(a, p, (int)tiles);
  }
}

moe_status launch_inner(const AdapterArgs& a, const AdapterParams& p, int sms) {
  if (p.slots == nullptr) {
    // four rows a warp share the loads of x; one row a warp where that leaves SMs without work
    const long long rows = (long long)a.T * a.rank;
    const bool wide = rows / 4 >= 8ll * sms * 2;
    const long long units = wide ? rows / 4 : rows;
    auto kernel = wide ? adapter_inner_dot_kernel<4> : adapter_inner_dot_kernel<1>;
    return launch_dependent(kernel, dim3((unsigned)((units + 7) / 8)), dim3(256), 0, a.stream, 1, p) == cudaSuccess ? MOE_OK
                                                                                                                    : MOE_ERR_CUDA;
  }
  const int r16 = (a.rank + 15) / 16 * 16, per_group = kInnerCols / r16;
  const int most = a.n_adapters < kAM ? a.n_adapters : kAM;
  const int groups = (most + per_group - 1) / per_group, blocks = token_blocks(a.T), ks = p.parts;
  CUtensorMap tm_x, tm_a;
  if (!make_tmap(&tm_x, a.x, (uint64_t)a.K, (uint64_t)a.T, 0, (uint64_t)a.K, 0, kAM) ||
      !make_tmap(&tm_a, a.A, (uint64_t)a.K, (uint64_t)a.rank, (uint64_t)a.n_adapters, (uint64_t)a.K, (uint64_t)a.rank * a.K,
                 (uint32_t)r16))
    return MOE_ERR_CUDA;
  const size_t smem = (size_t)kInnerStages * kInnerStageBytes + 1024;
  static PerDeviceOnce attr_set;
  if (!ensure_dynamic_smem(adapter_inner_umma_kernel, smem, attr_set)) return MOE_ERR_CUDA;
  return launch_dependent(adapter_inner_umma_kernel, dim3((unsigned)blocks, (unsigned)ks, (unsigned)groups), dim3(kInnerThreads),
                          smem, a.stream, (unsigned)ks, p, tm_x, tm_a, r16) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}

}  // namespace

size_t adapter_workspace_bytes(int T, int rank) {
  if (T <= kDotTokens) return align256((size_t)T * rank * 4);
  return vt_bytes(T, rank) + align256((size_t)pair_blocks(T) * sizeof(PairSlots)) +
         align256((size_t)pair_blocks(T) * kBadParts * (kPairM / 32) * 4);
}

moe_status launch_adapter_linear(const AdapterArgs& a) {
  const int sms = sm_count();
  if (sms <= 0) return MOE_ERR_CUDA;
  AdapterParams p{};
  p.T = a.T;
  p.K = a.K;
  p.M = a.M;
  p.n_adapters = a.n_adapters;
  p.rank = a.rank;
  p.k_per_sub = a.k_per_sub;
  p.swiglu_rows = a.swiglu_rows;
  p.x = a.x;
  p.A = a.A;
  p.B = a.B;
  p.scale = a.scale;
  p.adapter_id = a.adapter_id;
  p.y = a.y;
  p.dev_status = a.dev_status;
  unsigned char* ws = static_cast<unsigned char*>(a.ws);
  if (a.T <= kDotTokens) {
    p.v = reinterpret_cast<float*>(ws);
  } else {
    p.vt = reinterpret_cast<__nv_bfloat16*>(ws);
    ws += vt_bytes(a.T, a.rank);
    p.slots = reinterpret_cast<PairSlots*>(ws);
    ws += align256((size_t)pair_blocks(a.T) * sizeof(PairSlots));
    p.bad = reinterpret_cast<unsigned*>(ws);
    p.parts = cluster_size(token_blocks(a.T), (a.K + kABK - 1) / kABK, sms);   // one group of slots in most blocks
  }
  const moe_status r = launch_inner(a, p, sms);
  if (r != MOE_OK) return r;
  if (p.slots == nullptr) return a.swiglu_rows > 0 ? launch_few<true>(a, p, sms) : launch_few<false>(a, p, sms);
  return a.swiglu_rows > 0 ? launch_many<true>(a, p, sms) : launch_many<false>(a, p, sms);
}
