// Matrix products grouped by expert with ragged sizes, and the routed experts' backward pass made of them (formulas: allocmoe.h).
//
//   kRows     y  = x W_e^T    A = rows of x,   K-major;  B = W_e, K-major
//   kRowsT    dx = dy W_e     A = rows of dy,  K-major;  B = W_e, its columns contiguous: MN-major
//   kWeights  dW = dy^T x     A = dy, its columns contiguous: MN-major;  B = x, MN-major; the contraction runs over the ragged rows
//
// tcgen05 reads K-major and MN-major operands alike (two bits of the instruction descriptor), so no operand is ever transposed in
// memory and one kernel serves all three.  Bound by the tensor cores where a group has some hundred rows, by the weights' bytes
// (read or written once) where it has few.
//
// Persistent, one CTA an SM or one CTA pair a TPC (cta_group::2, M 256: half the bytes of B an SM).  Warp 0 issues TMA loads into a ring
// of stages of 64 along the contraction, warp 1 the products into one of two accumulators of 256 TMEM columns, warps 4..7 read the
// finished accumulator, round it and store it through shared memory with TMA (32 x 128-byte boxes, 128-byte swizzle, so neither the
// register-to-shared writes nor the stores conflict), while the next tile's products run.  Rows behind a segment's end belong to the
// next segment: a warp whose 32 rows are not all inside copies the valid ones out of shared memory itself.
//
// kWeights, ragged ends: the last block of 64 rows may hold rows of the next segment.  Products are issued for whole groups of 16
// rows only as far as the segment reaches; where the last group is not full, warp 2 zeroes its foreign rows in BOTH operands (a zero
// against another segment's NaN would still be NaN) before the stage is handed to the issuer.  Such a stage's loads complete on a
// barrier of its own CTA; the zeroing warp's arrival on the issuer's barrier takes the place of the load's.
// kWeights into fp32: the tensor core's accumulator truncates, so segments are cut into pieces of 512 rows, joined in
// global memory by TMA additions in fp32, in order.
#include <cuda.h>

#include "common.cuh"
#include "tmap.h"
#include "train.h"

namespace allocmoe {

constexpr int kGM = 128;                 // rows of the accumulator in one CTA
constexpr int kGN = 256;                 // columns of a tile
constexpr int kGK = 64;                  // contraction of a stage
constexpr int kGThreads = 256;
constexpr int kGABytes = kGM * kGK * 2;  // 16 KB
constexpr int kGMostStages = 6;
constexpr int kGMostGroups = 128;
constexpr int kGStageOut = 4096;         // a warp's staging buffer: 32 rows of 128 bytes; two a warp
constexpr int kGPiece = 512;             // rows that one fp32 accumulation takes
constexpr int kGBoxBytes = 64 * 64 * 2;  // an MN-major box: 64 columns of 64 rows

enum class GroupedOp { kRows, kRowsT, kWeights };

template <bool kPair>
struct GroupedRing {
  static constexpr int kBBytes = kGN * kGK * 2 / (kPair ? 2 : 1);
  static constexpr int kStageBytes = kGABytes + kBBytes;
  static constexpr int kStages = kPair ? 6 : 4;                       // 192 KB either way
  static constexpr size_t kBytes = (size_t)kStages * kStageBytes;
};

struct GroupedParams {
  const int32_t* offsets;
  int E, P;
  int n_cols;          // columns of the output
  int m_rows;          // kWeights: rows of the output of a group
  int k_len;           // kRows, kRowsT: length of the contraction
  int piece;           // kWeights: rows of one accumulation
  bool add;            // kWeights, fp32: add to what the output holds
  uint16_t* out;       // kRows, kRowsT: [P, n_cols]
  int32_t* dev_status;
};

struct GroupedMaps {
  CUtensorMap a[3];    // kRows, kRowsT: boxes of 128, 32 and 8 rows; kWeights: a[0] alone
  CUtensorMap b;
  CUtensorMap out;
};

struct GroupedCtl {
  uint64_t full[kGMostStages], empty[kGMostStages], tail[kGMostStages];
  uint64_t tmem_full[2], tmem_empty[2], drain;
  uint32_t tmem_base;
  volatile int abort_flag;
  volatile uint32_t progress;            // stages that the producer has filled
  int total_tiles;
  int row_start[kGMostGroups], row_end[kGMostGroups];
  int tile_start[kGMostGroups + 1];
};

// Segments clamped to [0, P] and to each other, and the tiles of each; `per_group` > 0: a fixed number of tiles for every group
// (kWeights), else blocks of tile_rows rows times n_blocks.  One warp.
DEV void grouped_table(GroupedCtl* ctl, const int32_t* offsets, int E, int P, int tile_rows, int n_blocks, int per_group, int32_t* dev_status) {
  const int lane = threadIdx.x & 31;
  int carry_row = 0, carry_tile = 0;
  for (int g0 = 0; g0 < E; g0 += 32) {
    const int g = g0 + lane;
    int at = g < E ? clamp_index(offsets[g], 0, P, dev_status) : 0;
    // a running maximum makes the list non-decreasing
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, at, d);
      if (lane >= d) at = max(at, o);
    }
    at = max(at, carry_row);
    int next = g < E ? clamp_index(offsets[g + 1], 0, P, dev_status) : 0;
    next = max(next, at);
    const int tiles = g < E ? (per_group > 0 ? per_group : (next - at + tile_rows - 1) / tile_rows * n_blocks) : 0;
    int incl = tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    if (g < E) {
      ctl->row_start[g] = at;
      ctl->row_end[g] = next;
      ctl->tile_start[g] = carry_tile + incl - tiles;
    }
    carry_row = __shfl_sync(0xffffffffu, at, 31);
    carry_tile += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (lane == 0) {
    ctl->tile_start[E] = carry_tile;
    ctl->total_tiles = carry_tile;
  }
}

struct GroupedTile {
  int e, m0, m_end;        // kRows, kRowsT: first row and the segment's end; kWeights: first output row and m_rows
  int n0;                  // first output column
  int k0, k_end;           // kWeights: the segment's rows
};

// Column blocks outermost, row blocks innermost: CTAs that run at the same time share a weight tile through L2.
template <GroupedOp kOp, int kTileM>
struct GroupedWalk {
  const GroupedCtl* c;
  int g = 0, n_blocks, m_blocks;
  DEV GroupedWalk(const GroupedCtl* ctl, const GroupedParams& p)
      : c(ctl), n_blocks((p.n_cols + kGN - 1) / kGN), m_blocks((p.m_rows + kTileM - 1) / kTileM) {}
  DEV GroupedTile at(int tile, const GroupedParams& p) {   // tile numbers never decrease
    while (tile >= c->tile_start[g + 1]) ++g;
    const int local = tile - c->tile_start[g], lo = c->row_start[g], hi = c->row_end[g];
    GroupedTile t;
    t.e = g;
    t.k0 = lo;
    t.k_end = hi;
    const int mb = kOp == GroupedOp::kWeights ? m_blocks : (hi - lo + kTileM - 1) / kTileM;
    t.n0 = local / mb * kGN;
    t.m0 = local % mb * kTileM + (kOp == GroupedOp::kWeights ? 0 : lo);
    t.m_end = kOp == GroupedOp::kWeights ? p.m_rows : hi;
    return t;
  }
};

// The blocks of 64 of one accumulation, and what the last one holds.
struct GroupedRun {
  int k0, blocks, last;    // kWeights: first row, blocks, rows in the last block
};
template <GroupedOp kOp>
DEV int grouped_pieces(const GroupedTile& t, const GroupedParams& p) {
  return kOp == GroupedOp::kWeights ? max(1, (t.k_end - t.k0 + p.piece - 1) / p.piece) : 1;
}
template <GroupedOp kOp>
DEV GroupedRun grouped_run(const GroupedTile& t, const GroupedParams& p, int piece) {
  if (kOp != GroupedOp::kWeights) return {0, (p.k_len + kGK - 1) / kGK, kGK};
  const int k0 = t.k0 + piece * p.piece, rows = min(p.piece, t.k_end - k0);
  const int blocks = (rows + kGK - 1) / kGK;
  return {k0, blocks, rows - (blocks - 1) * kGK};
}

template <bool kPair>
DEV void grouped_load_2d(void* dst, const void* map, uint64_t* bar, uint32_t cluster_bar, int c0, int c1) {
  if (kPair) tma_load_2d_pair(dst, map, cluster_bar, c0, c1); else tma_load_2d(dst, map, bar, c0, c1);
}
template <bool kPair>
DEV void grouped_load_3d(void* dst, const void* map, uint64_t* bar, uint32_t cluster_bar, int c0, int c1, int c2) {
  if (kPair) tma_load_3d_pair(dst, map, cluster_bar, c0, c1, c2); else tma_load_3d(dst, map, bar, c0, c1, c2);
}
template <bool kPair>
DEV void grouped_umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  if (kPair) umma_bf16_pair(d, a, b, idesc, acc); else umma_bf16(d, a, b, idesc, acc);
}
template <bool kPair>
DEV void grouped_commit(uint64_t* bar) {
  if (kPair) umma_commit_pair(bar, 3); else umma_commit(bar);
}

template <GroupedOp kOp, bool kPair, bool kF32>
__global__ void __launch_bounds__(kGThreads, 1)
grouped_kernel(const GroupedParams p, const __grid_constant__ GroupedMaps maps) {
  using Ring = GroupedRing<kPair>;
  constexpr int kTileM = kGM * (kPair ? 2 : 1), kStages = Ring::kStages, kStageBytes = Ring::kStageBytes, kBBytes = Ring::kBBytes;
  constexpr bool kW = kOp == GroupedOp::kWeights;
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
  unsigned char* staging = ring + Ring::kBytes;
  GroupedCtl& ctl = *reinterpret_cast<GroupedCtl*>(staging + 8 * kGStageOut);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = kPair ? cluster_cta_rank() : 0u;
  const int first_tile = kPair ? blockIdx.x >> 1 : blockIdx.x, tile_step = kPair ? gridDim.x >> 1 : gridDim.x;

  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(&ctl.full[s], kPair ? 2 : 1); mbar_init(&ctl.empty[s], 1); mbar_init(&ctl.tail[s], 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(&ctl.tmem_full[a], 1); mbar_init(&ctl.tmem_empty[a], kPair ? 8 : 4); }
    mbar_init(&ctl.drain, 1);
    ctl.abort_flag = 0;
    ctl.progress = 0;
    fence_barrier_init();
    prefetch_tensormap(&maps.a[0]);
    prefetch_tensormap(&maps.b);
    prefetch_tensormap(&maps.out);
  }
  if (warp == 1) {
    if (kPair) { tmem_alloc_pair(&ctl.tmem_base, 512); tmem_relinquish_pair(); }
    else { tmem_alloc(&ctl.tmem_base, 512); tmem_relinquish(); }
  }
  pdl_prologue_done();
  if (warp == 2) {
    const int n_blocks = (p.n_cols + kGN - 1) / kGN;
    grouped_table(&ctl, p.offsets, p.E, p.P, kTileM, n_blocks, kW ? n_blocks * ((p.m_rows + kTileM - 1) / kTileM) : 0, p.dev_status);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (kPair) cluster_sync_all();        // both CTAs' barriers are initialised before either signals the other
  tc_fence_after_sync();
  const uint32_t tmem_base = ctl.tmem_base;
  const int total_tiles = ctl.total_tiles;
  volatile int* abort_flag = &ctl.abort_flag;

  if (warp == 0) {
    // ======================= loads (each CTA its own part) =======================
    if (elect_one()) {
      GroupedWalk<kOp, kTileM> walk(&ctl, p);
      uint32_t it = 0, s = 0, ph = 0, tail_used = 0, tail_ph = 0;   // tail_*: a bit a stage
      bool ok = true;
      for (int tile = first_tile; ok && tile < total_tiles; tile += tile_step) {
        const GroupedTile t = walk.at(tile, p);
        const int m0 = t.m0 + (int)rank * kGM, n0 = t.n0 + (int)rank * (kGN / 2);
        // rows of A that the tile has: the smallest box that covers them; the accumulator's other rows are never stored
        const int valid = min(max(t.m_end - m0, 0), kGM);
        const int box = valid > 32 ? 0 : valid > 8 ? 1 : 2;
        const uint32_t a_bytes = kW ? kGABytes : valid > 0 ? (box == 0 ? 128 : box == 1 ? 32 : 8) * (kGK * 2) : 0;
        const int pieces = grouped_pieces<kOp>(t, p);
        for (int piece = 0; ok && piece < pieces; ++piece) {
          const GroupedRun run = grouped_run<kOp>(t, p, piece);
          for (int kb = 0; kb < run.blocks; ++kb) {
            if (!(ok = mbar_wait_bounded(&ctl.empty[s], ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
            unsigned char* sa = ring + s * kStageBytes;
            unsigned char* sb = sa + kGABytes;
            uint64_t* bar = &ctl.full[s];
            const uint32_t cluster_bar = kPair ? cluster_addr_of(bar, 0) : 0u;
            if constexpr (kW) {
              const bool fix = kb == run.blocks - 1 && (run.last & 15) != 0;
              const int row = run.k0 + kb * kGK;
              tail_used = (tail_used & ~(1u << s)) | ((fix ? 1u : 0u) << s);
              if (fix) {     // lands in this CTA's own barrier; the zeroing warp hands the stage on
                mbar_expect_tx(&ctl.tail[s], kStageBytes);
                for (int j = 0; j < kGM / 64; ++j) tma_load_2d(sa + j * kGBoxBytes, &maps.a[0], &ctl.tail[s], m0 + j * 64, row);
                for (int j = 0; j < kBBytes / kGBoxBytes; ++j) tma_load_2d(sb + j * kGBoxBytes, &maps.b, &ctl.tail[s], n0 + j * 64, row);
                tail_ph ^= 1u << s;
              } else {
                if (kPair) mbar_expect_tx_cluster(cluster_bar, kStageBytes); else mbar_expect_tx(bar, kStageBytes);
                for (int j = 0; j < kGM / 64; ++j) grouped_load_2d<kPair>(sa + j * kGBoxBytes, &maps.a[0], bar, cluster_bar, m0 + j * 64, row);
                for (int j = 0; j < kBBytes / kGBoxBytes; ++j) grouped_load_2d<kPair>(sb + j * kGBoxBytes, &maps.b, bar, cluster_bar, n0 + j * 64, row);
              }
            } else {
              if (kPair) mbar_expect_tx_cluster(cluster_bar, a_bytes + kBBytes); else mbar_expect_tx(bar, a_bytes + kBBytes);
              if (a_bytes != 0) grouped_load_2d<kPair>(sa, &maps.a[box], bar, cluster_bar, kb * kGK, m0);
              if constexpr (kOp == GroupedOp::kRows) {
                grouped_load_3d<kPair>(sb, &maps.b, bar, cluster_bar, kb * kGK, n0, t.e);
              } else {
                for (int j = 0; j < kBBytes / kGBoxBytes; ++j)
                  grouped_load_3d<kPair>(sb + j * kGBoxBytes, &maps.b, bar, cluster_bar, n0 + j * 64, kb * kGK, t.e);
              }
            }
            ctl.progress = ++it;
            if (++s == kStages) { s = 0; ph ^= 1u; }
          }
        }
      }
      // every load must have landed before the CTA may leave.  The peer's loads complete on the leader's barriers; it learns of
      // them through `empty`.
      for (uint32_t q = it > (uint32_t)kStages ? it - kStages : 0u; q < it; ++q) {
        const uint32_t st = q % kStages, par = (q / kStages) & 1u;
        if (kW && (tail_used >> st & 1u)) mbar_wait_drain(&ctl.tail[st], (tail_ph >> st & 1u) ^ 1u);
        else if (rank == 0) mbar_wait_drain(&ctl.full[st], par);
        else mbar_wait_drain(&ctl.empty[st], par);
      }
    }
  } else if (warp == 1) {
    // ======================= products (the leader alone) =======================
    if (rank == 0 && elect_one()) {
      GroupedWalk<kOp, kTileM> walk(&ctl, p);
      constexpr uint32_t idesc = umma_idesc_bf16(kTileM, kGN) | (kW ? 1u << 15 : 0u) | (kOp != GroupedOp::kRows ? 1u << 16 : 0u);
      constexpr uint32_t kStepA = kW ? 128 : 2, kStepB = kOp != GroupedOp::kRows ? 128 : 2;   // 16 along the contraction, in 16 bytes
      uint32_t s = 0, ph = 0, acc = 0;
      bool ok = true;
      for (int tile = first_tile; ok && tile < total_tiles; tile += tile_step) {
        const GroupedTile t = walk.at(tile, p);
        const int pieces = grouped_pieces<kOp>(t, p);
        for (int piece = 0; ok && piece < pieces; ++piece, ++acc) {
          const GroupedRun run = grouped_run<kOp>(t, p, piece);
          const uint32_t a = acc & 1u, aph = (acc >> 1) & 1u;
          if (!(ok = mbar_wait_bounded(&ctl.tmem_empty[a], aph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
          tc_fence_after_sync();
          const uint32_t d = tmem_base + a * kGN;
          for (int kb = 0; kb < run.blocks; ++kb) {
            const int rows = kW && kb == run.blocks - 1 ? run.last : kGK;
            if (kW && kPair && (rows & 15) != 0)    // both CTAs' zeroing warps wrote operands of these products
              ok = mbar_wait_acquire_cluster(&ctl.full[s], ph, abort_flag, p.dev_status, kWaitLimitClk);
            else
              ok = mbar_wait_bounded(&ctl.full[s], ph, abort_flag, p.dev_status, kWaitLimitClk);
            if (!ok) break;
            tc_fence_after_sync();
            const uint32_t sa = smem_u32(ring + s * kStageBytes), sb = sa + kGABytes;
            const uint64_t da = kW ? umma_desc_mn_sw128(sa, kGBoxBytes) : umma_desc_sw128(sa);
            const uint64_t db = kOp != GroupedOp::kRows ? umma_desc_mn_sw128(sb, kGBoxBytes) : umma_desc_sw128(sb);
            if (kW && rows < kGK) {
              for (int k = 0; k * 16 < rows; ++k)
                grouped_umma<kPair>(d, da + (uint64_t)(k * kStepA), db + (uint64_t)(k * kStepB), idesc, (kb | k) != 0 ? 1u : 0u);
            } else {
#pragma unroll
              for (int k = 0; k < kGK / 16; ++k)
                grouped_umma<kPair>(d, da + (uint64_t)(k * kStepA), db + (uint64_t)(k * kStepB), idesc, (kb | k) != 0 ? 1u : 0u);
            }
            grouped_commit<kPair>(&ctl.empty[s]);
            if (++s == kStages) { s = 0; ph ^= 1u; }
          }
          if (ok) grouped_commit<kPair>(&ctl.tmem_full[a]);
        }
      }
      if (kPair) umma_commit_pair(&ctl.drain, 1); else umma_commit(&ctl.drain);
      mbar_wait_drain(&ctl.drain, 0u);       // every product is complete before TMEM is freed
    }
  } else if (kW && warp == 2) {
    // ======================= foreign rows of the last block zeroed (each CTA its own part) =======================
    GroupedWalk<kOp, kTileM> walk(&ctl, p);
    uint32_t it = 0, tail_ph = 0;
    bool ok = true;
    for (int tile = first_tile; ok && tile < total_tiles; tile += tile_step) {
      const GroupedTile t = walk.at(tile, p);
      const int pieces = grouped_pieces<kOp>(t, p);
      for (int piece = 0; piece < pieces; ++piece) {
        const GroupedRun run = grouped_run<kOp>(t, p, piece);
        it += run.blocks;
        if (run.blocks == 0 || (run.last & 15) == 0) continue;
        const uint32_t s = (it - 1) % kStages;
        if (!(ok = mbar_spin_progress_warp(&ctl.tail[s], tail_ph >> s & 1u, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk))) break;
        tail_ph ^= 1u << s;
        unsigned char* stage = ring + s * kStageBytes;
        const int from = run.last, to = (run.last + 15) & ~15;
        for (int i = lane; i < (kStageBytes / kGBoxBytes) * 8 * (to - from); i += 32) {
          const int piece16 = i & 7, box = (i >> 3) % (kStageBytes / kGBoxBytes), row = from + (i >> 3) / (kStageBytes / kGBoxBytes);
          *reinterpret_cast<uint4*>(stage + box * kGBoxBytes + row * 128 + piece16 * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (kPair) mbar_arrive_release_cluster(cluster_addr_of(&ctl.full[s], 0)); else mbar_arrive(&ctl.full[s]);
        }
      }
    }
  } else if (warp >= 4) {
    // ======================= results =======================
    GroupedWalk<kOp, kTileM> walk(&ctl, p);
    const int q = warp & 3;
    unsigned char* mine = staging + q * 2 * kGStageOut;
    constexpr int kCols = kF32 ? 32 : 64;      // columns of a 128-byte row
    const bool issuer = elect_one();
    uint32_t acc = 0, turn = 0;
    bool ok = true;
    for (int tile = first_tile; ok && tile < total_tiles; tile += tile_step) {
      const GroupedTile t = walk.at(tile, p);
      const int pieces = grouped_pieces<kOp>(t, p);
      const int row0 = t.m0 + (int)rank * kGM + q * 32;
      for (int piece = 0; piece < pieces; ++piece, ++acc) {
        const GroupedRun run = grouped_run<kOp>(t, p, piece);
        const uint32_t a = acc & 1u, aph = (acc >> 1) & 1u;
        if (!(ok = mbar_spin_progress_warp(&ctl.tmem_full[a], aph, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk))) break;
        tc_fence_after_sync();
        const bool add = kF32 && (p.add || piece > 0);
        // an addition to what this thread has stored before: those stores are complete first
        if (kF32 && piece > 0 && issuer) bulk_wait_all();
        const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + a * kGN;
        const int n_cols = row0 < t.m_end && !(run.blocks == 0 && add) ? min(kGN, p.n_cols - t.n0) : 0;
#pragma unroll 1
        for (int c = 0; c < n_cols; c += kCols) {
          uint32_t v[kCols / 32][32];
          if (run.blocks > 0) {
#pragma unroll
            for (int h = 0; h < kCols / 32; ++h) tmem_ld_32x32(taddr + c + h * 32, v[h]);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int h = 0; h < kCols / 32; ++h)
#pragma unroll
              for (int i = 0; i < 32; ++i) v[h][i] = 0u;
          }
          unsigned char* buf = mine + (turn++ & 1) * kGStageOut;
          if (issuer) bulk_wait_read<1>();       // the store before last has left this buffer
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            uint4 w;
            if constexpr (kF32) {
              w = make_uint4(v[0][4 * j], v[0][4 * j + 1], v[0][4 * j + 2], v[0][4 * j + 3]);
            } else {
              const uint32_t* u = v[j >> 2] + (j & 3) * 8;
              w = make_uint4(pack_bf16x2(__uint_as_float(u[0]), __uint_as_float(u[1])), pack_bf16x2(__uint_as_float(u[2]), __uint_as_float(u[3])),
                             pack_bf16x2(__uint_as_float(u[4]), __uint_as_float(u[5])), pack_bf16x2(__uint_as_float(u[6]), __uint_as_float(u[7])));
            }
            *reinterpret_cast<uint4*>(buf + lane * 128 + ((j ^ (lane & 7)) << 4)) = w;
          }
          if (kW || row0 + 32 <= t.m_end) {
            fence_proxy_async_smem();
            __syncwarp();
            if (issuer) {
              if (!kW) tma_store_2d(buf, &maps.out, t.n0 + c, row0);
              else if (add) tma_add_3d(buf, &maps.out, t.n0 + c, row0, t.e);
              else tma_store_3d(buf, &maps.out, t.n0 + c, row0, t.e);
              bulk_commit();
            }
          } else {
            __syncwarp();
            const int j = lane & 7, col = t.n0 + c + j * 8;
            for (int r = lane >> 3; r < t.m_end - row0; r += 4)
              if (col < p.n_cols)
                *reinterpret_cast<uint4*>(p.out + (size_t)(row0 + r) * p.n_cols + col) = *reinterpret_cast<const uint4*>(buf + r * 128 + ((j ^ (r & 7)) << 4));
            if (issuer) bulk_commit();           // an empty group keeps the count of stores in step with the buffers
            __syncwarp();
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          if (kPair) mbar_arrive_cluster(cluster_addr_of(&ctl.tmem_empty[a], 0)); else mbar_arrive(&ctl.tmem_empty[a]);
        }
      }
    }
    if (issuer) bulk_wait_all();
  }

  tc_fence_before_sync();
  __syncthreads();
  if (kPair) cluster_sync_all();      // neither CTA leaves (or frees TMEM) while its peer may still touch it
  if (warp == 1) {
    __syncwarp();
    tc_fence_after_sync();
    if (kPair) tmem_dealloc_pair(tmem_base, 512); else tmem_dealloc(tmem_base, 512);
  }
}

// ------------------------------------------------------------------------------------------------
// The experts' backward pass up to their hidden layer, in one launch: u = x W13_e^T computed again, dh = dy W2_e, and from both
// h, du1 and du3 (formulas: allocmoe.h).  A tile is kTileM rows of an expert times 128 hidden columns: first dh into 128 TMEM columns
// (W2_e as MN-major B operand), then u1 and u3 into 256.  dh has two places that take turns, so the products of the next tile's dh
// run while this tile's three accumulators are read: 512 columns in all.  Nothing of u or dh touches memory.
constexpr int kDuCols = 128;

struct DuParams {
  const int32_t* offsets;
  int E, P, H, I;
  uint16_t* h;         // [P, I]
  uint16_t* du;        // [P, 2I]
  int32_t* dev_status;
};
struct DuMaps {
  CUtensorMap x[3], dy[3];     // boxes of 128, 32 and 8 rows
  CUtensorMap w13, w2;
};
struct DuCtl {
  uint64_t full[kGMostStages], empty[kGMostStages];
  uint64_t tmem_full, u_empty, dh_empty[2], drain;
  uint32_t tmem_base;
  volatile int abort_flag;
  volatile uint32_t progress;
  // the tables of GroupedCtl
  GroupedCtl table;
};

template <bool kPair>
__global__ void __launch_bounds__(kGThreads, 1)
expert_du_kernel(const DuParams p, const __grid_constant__ DuMaps maps) {
  using Ring = GroupedRing<kPair>;
  constexpr int kTileM = kGM * (kPair ? 2 : 1), kStages = Ring::kStages, kStageBytes = Ring::kStageBytes, kBBytes = Ring::kBBytes;
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
  DuCtl& ctl = *reinterpret_cast<DuCtl*>(ring + Ring::kBytes);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = kPair ? cluster_cta_rank() : 0u;
  const int first_tile = kPair ? blockIdx.x >> 1 : blockIdx.x, tile_step = kPair ? gridDim.x >> 1 : gridDim.x;
  const int blocks = p.H / kGK, n_blocks = (p.I + kDuCols - 1) / kDuCols;

  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(&ctl.full[s], kPair ? 2 : 1); mbar_init(&ctl.empty[s], 1); }
    mbar_init(&ctl.tmem_full, 1);
    mbar_init(&ctl.u_empty, kPair ? 8 : 4);
    for (int a = 0; a < 2; ++a) mbar_init(&ctl.dh_empty[a], kPair ? 8 : 4);
    mbar_init(&ctl.drain, 1);
    ctl.abort_flag = 0;
    ctl.progress = 0;
    fence_barrier_init();
    prefetch_tensormap(&maps.x[0]);
    prefetch_tensormap(&maps.dy[0]);
    prefetch_tensormap(&maps.w13);
    prefetch_tensormap(&maps.w2);
  }
  if (warp == 1) {
    if (kPair) { tmem_alloc_pair(&ctl.tmem_base, 512); tmem_relinquish_pair(); }
    else { tmem_alloc(&ctl.tmem_base, 512); tmem_relinquish(); }
  }
  pdl_prologue_done();
  if (warp == 2) grouped_table(&ctl.table, p.offsets, p.E, p.P, kTileM, n_blocks, 0, p.dev_status);
  tc_fence_before_sync();
  __syncthreads();
  if (kPair) cluster_sync_all();
  tc_fence_after_sync();
  const uint32_t tmem_base = ctl.tmem_base;
  const int total_tiles = ctl.table.total_tiles;
  volatile int* abort_flag = &ctl.abort_flag;
  int g = 0;
  auto tile_at = [&](int tile) {
    while (tile >= ctl.table.tile_start[g + 1]) ++g;
    const int local = tile - ctl.table.tile_start[g], lo = ctl.table.row_start[g], hi = ctl.table.row_end[g];
    const int mb = (hi - lo + kTileM - 1) / kTileM;
    GroupedTile t;
    t.e = g;
    t.n0 = local / mb * kDuCols;
    t.m0 = lo + local % mb * kTileM;
    t.m_end = hi;
    t.k0 = t.k_end = 0;
    return t;
  };

  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0, s = 0, ph = 0;
      bool ok = true;
      for (int tile = first_tile; ok && tile < total_tiles; tile += tile_step) {
        const GroupedTile t = tile_at(tile);
        const int m0 = t.m0 + (int)rank * kGM, valid = min(max(t.m_end - m0, 0), kGM);
        const int box = valid > 32 ? 0 : valid > 8 ? 1 : 2;
        const uint32_t a_bytes = valid > 0 ? (box == 0 ? 128 : box == 1 ? 32 : 8) * (kGK * 2) : 0;
        for (int phase = 0; ok && phase < 2; ++phase) {       // dh, then u
          const CUtensorMap* ma = phase == 0 ? &maps.dy[box] : &maps.x[box];
          const uint32_t b_bytes = phase == 0 ? kBBytes / 2 : kBBytes;
          for (int kb = 0; kb < blocks; ++kb) {
            if (!(ok = mbar_wait_bounded(&ctl.empty[s], ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
            unsigned char* sa = ring + s * kStageBytes;
            unsigned char* sb = sa + kGABytes;
            uint64_t* bar = &ctl.full[s];
            const uint32_t cluster_bar = kPair ? cluster_addr_of(bar, 0) : 0u;
            if (kPair) mbar_expect_tx_cluster(cluster_bar, a_bytes + b_bytes); else mbar_expect_tx(bar, a_bytes + b_bytes);
            if (a_bytes != 0) grouped_load_2d<kPair>(sa, ma, bar, cluster_bar, kb * kGK, m0);
            if (phase == 0) {
              for (int j = 0; j < kDuCols / 64 / (kPair ? 2 : 1); ++j)
                grouped_load_3d<kPair>(sb + j * kGBoxBytes, &maps.w2, bar, cluster_bar, t.n0 + (int)rank * 64 + j * 64, kb * kGK, t.e);
            } else if (kPair) {                               // leader W1's rows, peer W3's
              grouped_load_3d<kPair>(sb, &maps.w13, bar, cluster_bar, kb * kGK, (int)rank * p.I + t.n0, t.e);
            } else {
              grouped_load_3d<kPair>(sb, &maps.w13, bar, cluster_bar, kb * kGK, t.n0, t.e);
              grouped_load_3d<kPair>(sb + kBBytes / 2, &maps.w13, bar, cluster_bar, kb * kGK, p.I + t.n0, t.e);
            }
            ctl.progress = ++it;
            if (++s == kStages) { s = 0; ph ^= 1u; }
          }
        }
      }
      for (uint32_t q = it > (uint32_t)kStages ? it - kStages : 0u; q < it; ++q)
        mbar_wait_drain(rank == 0 ? &ctl.full[q % kStages] : &ctl.empty[q % kStages], (q / kStages) & 1u);
    }
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) {
      constexpr uint32_t idesc_dh = umma_idesc_bf16(kTileM, kDuCols) | 1u << 16, idesc_u = umma_idesc_bf16(kTileM, 2 * kDuCols);
      uint32_t s = 0, ph = 0, n = 0;
      bool ok = true;
      for (int tile = first_tile; ok && tile < total_tiles; tile += tile_step, ++n) {
        for (int phase = 0; ok && phase < 2; ++phase) {
          if (phase == 0) ok = mbar_wait_bounded(&ctl.dh_empty[n & 1u], ((n >> 1) & 1u) ^ 1u, abort_flag, p.dev_status, kWaitLimitClk);
          else ok = mbar_wait_bounded(&ctl.u_empty, (n & 1u) ^ 1u, abort_flag, p.dev_status, kWaitLimitClk);
          if (!ok) break;
          tc_fence_after_sync();
          const uint32_t d = tmem_base + (phase == 0 ? (n & 1u) * kDuCols : 2 * kDuCols);
          for (int kb = 0; kb < blocks; ++kb) {
            if (!(ok = mbar_wait_bounded(&ctl.full[s], ph, abort_flag, p.dev_status, kWaitLimitClk))) break;
            tc_fence_after_sync();
            const uint32_t sa = smem_u32(ring + s * kStageBytes), sb = sa + kGABytes;
            const uint64_t da = umma_desc_sw128(sa);
            if (phase == 0) {
              const uint64_t db = umma_desc_mn_sw128(sb, kGBoxBytes);
#pragma unroll
              for (int k = 0; k < kGK / 16; ++k) grouped_umma<kPair>(d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 128), idesc_dh, (kb | k) != 0 ? 1u : 0u);
            } else {
              const uint64_t db = umma_desc_sw128(sb);
#pragma unroll
              for (int k = 0; k < kGK / 16; ++k) grouped_umma<kPair>(d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc_u, (kb | k) != 0 ? 1u : 0u);
            }
            grouped_commit<kPair>(&ctl.empty[s]);
            if (++s == kStages) { s = 0; ph ^= 1u; }
          }
        }
        if (ok) grouped_commit<kPair>(&ctl.tmem_full);
      }
      if (kPair) umma_commit_pair(&ctl.drain, 1); else umma_commit(&ctl.drain);
      mbar_wait_drain(&ctl.drain, 0u);
    }
  } else if (warp >= 4) {
    const int q = warp & 3;
    uint32_t n = 0;
    for (int tile = first_tile; tile < total_tiles; tile += tile_step, ++n) {
      const GroupedTile t = tile_at(tile);
      if (!mbar_spin_progress_warp(&ctl.tmem_full, n & 1u, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk)) break;
      tc_fence_after_sync();
      const int row0 = t.m0 + (int)rank * kGM + q * 32, row = row0 + lane;
      const uint32_t lanes = tmem_base + ((uint32_t)(q * 32) << 16), t_dh = lanes + (n & 1u) * kDuCols, t_u = lanes + 2 * kDuCols;
      const int n_cols = row0 < t.m_end ? min(kDuCols, p.I - t.n0) : 0;     // I is a multiple of 64
#pragma unroll 1
      for (int c = 0; c < n_cols; c += 32) {
        uint32_t d[32], u1[32], u3[32];
        tmem_ld_32x32(t_dh + c, d);
        tmem_ld_32x32(t_u + c, u1);
        tmem_ld_32x32(t_u + kDuCols + c, u3);
        tmem_ld_wait();
        uint32_t ph[16], p1[16], p3[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float h[2], d1[2], d3[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float a = __uint_as_float(u1[2 * i + k]), b = __uint_as_float(u3[2 * i + k]), dh = __uint_as_float(d[2 * i + k]);
            const float den = 1.f + __expf(-a), sg = __fdividef(1.f, den), s = a * sg;
            h[k] = __fdividef(a * b, den);           // the forward pass's h, to the bit
            d3[k] = dh * s;
            d1[k] = dh * b * (sg * (1.f + a * (1.f - sg)));
          }
          ph[i] = pack_bf16x2(h[0], h[1]);
          p1[i] = pack_bf16x2(d1[0], d1[1]);
          p3[i] = pack_bf16x2(d3[0], d3[1]);
        }
        if (row < t.m_end) {
          uint4* oh = reinterpret_cast<uint4*>(p.h + (size_t)row * p.I + t.n0 + c);
          uint4* o1 = reinterpret_cast<uint4*>(p.du + (size_t)row * 2 * p.I + t.n0 + c);
          uint4* o3 = reinterpret_cast<uint4*>(p.du + (size_t)row * 2 * p.I + p.I + t.n0 + c);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            oh[i] = make_uint4(ph[4 * i], ph[4 * i + 1], ph[4 * i + 2], ph[4 * i + 3]);
            o1[i] = make_uint4(p1[4 * i], p1[4 * i + 1], p1[4 * i + 2], p1[4 * i + 3]);
            o3[i] = make_uint4(p3[4 * i], p3[4 * i + 1], p3[4 * i + 2], p3[4 * i + 3]);
          }
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        if (kPair) {
          mbar_arrive_cluster(cluster_addr_of(&ctl.dh_empty[n & 1u], 0));
          mbar_arrive_cluster(cluster_addr_of(&ctl.u_empty, 0));
        } else {
          mbar_arrive(&ctl.dh_empty[n & 1u]);
          mbar_arrive(&ctl.u_empty);
        }
      }
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (kPair) cluster_sync_all();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after_sync();
    if (kPair) tmem_dealloc_pair(tmem_base, 512); else tmem_dealloc(tmem_base, 512);
  }
}

}  // namespace allocmoe

using namespace allocmoe;

namespace {

PerDeviceInt g_sms;
int sm_count() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 148;
  int n = g_sms.get(dev);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 148;
    g_sms.set(dev, n);
  }
  return n;
}

template <GroupedOp kOp, bool kPair, bool kF32>
moe_status launch_variant(const GroupedParams& p, const GroupedMaps& m, cudaStream_t stream) {
  constexpr size_t smem = GroupedRing<kPair>::kBytes + 8 * kGStageOut + sizeof(GroupedCtl) + 1024;
  static_assert(smem <= 232448, "ring, staging and control block exceed the 227 KB a CTA may use");
  static PerDeviceOnce attr_set;
  auto kernel = grouped_kernel<kOp, kPair, kF32>;
  if (!ensure_dynamic_smem(kernel, smem, attr_set)) return MOE_ERR_CUDA;
  const unsigned grid = (unsigned)(kPair ? sm_count() & ~1 : sm_count());
  return launch_dependent_cluster(kernel, dim3(grid), dim3(kGThreads), smem, stream, dim3(kPair ? 2 : 1, 1, 1), p, m) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}

bool row_maps(CUtensorMap (&m)[3], const void* base, uint64_t cols, uint64_t rows) {
  return make_tmap(&m[0], base, cols, rows, 0, cols, 0, 128) && make_tmap(&m[1], base, cols, rows, 0, cols, 0, 32) &&
         make_tmap(&m[2], base, cols, rows, 0, cols, 0, 8);
}

// A pair's tile is 256 rows of a group: used where the groups have more than 128 on average.
bool pair_rows(int64_t rows, int groups) { return rows > 128ll * groups; }

// y [P, n] = rows [P, k] times W_e: kRows W [E, n, k], kRowsT W [E, k, n]
template <GroupedOp kOp>
moe_status launch_rows(int P, int k, int n, int E, const uint16_t* rows, const int32_t* offsets, const uint16_t* W, uint16_t* out,
                       int32_t* dev_status, cudaStream_t stream) {
  const bool pair = pair_rows(P, E);
  GroupedMaps m;
  bool ok = row_maps(m.a, rows, (uint64_t)k, (uint64_t)P);
  if (kOp == GroupedOp::kRows) ok = ok && make_tmap(&m.b, W, (uint64_t)k, (uint64_t)n, (uint64_t)E, (uint64_t)k, (uint64_t)n * k, pair ? 128 : 256);
  else ok = ok && make_tmap(&m.b, W, (uint64_t)n, (uint64_t)k, (uint64_t)E, (uint64_t)n, (uint64_t)n * k, 64);
  ok = ok && make_tmap(&m.out, out, (uint64_t)n, (uint64_t)P, 0, (uint64_t)n, 0, 32);
  if (!ok) return MOE_ERR_CUDA;
  GroupedParams p{};
  p.offsets = offsets;
  p.E = E;
  p.P = P;
  p.n_cols = n;
  p.k_len = k;
  p.out = out;
  p.dev_status = dev_status;
  return pair ? launch_variant<kOp, true, false>(p, m, stream) : launch_variant<kOp, false, false>(p, m, stream);
}

// dW [E, m, n] = a^T b over the rows of each segment; a [P, m], b [P, n]
moe_status launch_weights(int P, int mm, int n, int E, const uint16_t* a, const uint16_t* b, const int32_t* offsets, void* dW, bool f32, bool add,
                          int32_t* dev_status, cudaStream_t stream) {
  GroupedMaps m;
  bool ok = make_tmap(&m.a[0], a, (uint64_t)mm, (uint64_t)P, 0, (uint64_t)mm, 0, 64);
  m.a[1] = m.a[2] = m.a[0];
  ok = ok && make_tmap(&m.b, b, (uint64_t)n, (uint64_t)P, 0, (uint64_t)n, 0, 64);
  if (f32) ok = ok && make_tmap_f32(&m.out, dW, (uint64_t)n, (uint64_t)mm, (uint64_t)E, 32);
  else ok = ok && make_tmap(&m.out, dW, (uint64_t)n, (uint64_t)mm, (uint64_t)E, (uint64_t)n, (uint64_t)n * mm, 32);
  if (!ok) return MOE_ERR_CUDA;
  GroupedParams p{};
  p.offsets = offsets;
  p.E = E;
  p.P = P;
  p.n_cols = n;
  p.m_rows = mm;
  p.piece = f32 ? kGPiece : 1 << 30;
  p.add = add;
  p.dev_status = dev_status;
  if (mm > kGM) return f32 ? launch_variant<GroupedOp::kWeights, true, true>(p, m, stream) : launch_variant<GroupedOp::kWeights, true, false>(p, m, stream);
  return f32 ? launch_variant<GroupedOp::kWeights, false, true>(p, m, stream) : launch_variant<GroupedOp::kWeights, false, false>(p, m, stream);
}

template <bool kPair>
moe_status launch_du(const DuParams& p, const DuMaps& m, cudaStream_t stream) {
  constexpr size_t smem = GroupedRing<kPair>::kBytes + sizeof(DuCtl) + 1024;
  static_assert(smem <= 232448, "ring and control block exceed the 227 KB a CTA may use");
  static PerDeviceOnce attr_set;
  if (!ensure_dynamic_smem(expert_du_kernel<kPair>, smem, attr_set)) return MOE_ERR_CUDA;
  const unsigned grid = (unsigned)(kPair ? sm_count() & ~1 : sm_count());
  return launch_dependent_cluster(expert_du_kernel<kPair>, dim3(grid), dim3(kGThreads), smem, stream, dim3(kPair ? 2 : 1, 1, 1), p, m) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}

}  // namespace

moe_status launch_grouped_gemm(const moe_grouped_shape* s, const uint16_t* x, const int32_t* offsets, const uint16_t* W, uint16_t* y,
                               int32_t* dev_status, cudaStream_t stream) {
  return launch_rows<GroupedOp::kRows>(s->P, s->K, s->M, s->E, x, offsets, W, y, dev_status, stream);
}
moe_status launch_grouped_gemm_dx(const moe_grouped_shape* s, const uint16_t* dy, const int32_t* offsets, const uint16_t* W, uint16_t* dx,
                                  int32_t* dev_status, cudaStream_t stream) {
  return launch_rows<GroupedOp::kRowsT>(s->P, s->M, s->K, s->E, dy, offsets, W, dx, dev_status, stream);
}
moe_status launch_grouped_gemm_dw(const moe_grouped_shape* s, const uint16_t* dy, const uint16_t* x, const int32_t* offsets, void* dW,
                                  int32_t* dev_status, cudaStream_t stream) {
  return launch_weights(s->P, s->M, s->K, s->E, dy, x, offsets, dW, (s->flags & MOE_GROUPED_DW_FP32) != 0, (s->flags & MOE_GROUPED_DW_ADD) != 0,
                        dev_status, stream);
}

moe_status launch_ffn_backward(const FfnBackwardArgs& a) {
  const moe_shape* s = a.s;
  const size_t w = (size_t)s->N * s->H * s->I * 2;
  if (a.budget == 0) {      // no pairs: the weights' gradients are zero
    if (a.dW13 != nullptr && cudaMemsetAsync(a.dW13, 0, 2 * w, a.stream) != cudaSuccess) return MOE_ERR_CUDA;
    if (a.dW2 != nullptr && cudaMemsetAsync(a.dW2, 0, w, a.stream) != cudaSuccess) return MOE_ERR_CUDA;
    return MOE_OK;
  }
  const int P = (int)a.budget, H = s->H, I = s->I, N = s->N;
  const bool pair = pair_rows(P, N);
  DuMaps m;
  bool ok = row_maps(m.x, a.x_perm, (uint64_t)H, (uint64_t)P) && row_maps(m.dy, a.d_y, (uint64_t)H, (uint64_t)P);
  ok = ok && make_tmap(&m.w13, a.W13, (uint64_t)H, 2ull * I, (uint64_t)N, (uint64_t)H, 2ull * I * H, kDuCols);
  ok = ok && make_tmap(&m.w2, a.W2, (uint64_t)I, (uint64_t)H, (uint64_t)N, (uint64_t)I, (uint64_t)H * I, 64);
  if (!ok) return MOE_ERR_CUDA;
  DuParams p{};
  p.offsets = a.expert_offsets;
  p.E = N;
  p.P = P;
  p.H = H;
  p.I = I;
  p.h = a.h;
  p.du = a.du;
  p.dev_status = a.dev_status;
  moe_status r = pair ? launch_du<true>(p, m, a.stream) : launch_du<false>(p, m, a.stream);
  if (r == MOE_OK && a.dW2 != nullptr) r = launch_weights(P, H, I, N, a.d_y, a.h, a.expert_offsets, a.dW2, false, false, a.dev_status, a.stream);
  if (r == MOE_OK && a.dx != nullptr) r = launch_rows<GroupedOp::kRowsT>(P, 2 * I, H, N, a.du, a.expert_offsets, a.W13, a.dx, a.dev_status, a.stream);
  if (r == MOE_OK && a.dW13 != nullptr) r = launch_weights(P, 2 * I, H, N, a.du, a.x_perm, a.expert_offsets, a.dW13, false, false, a.dev_status, a.stream);
  return r;
}
