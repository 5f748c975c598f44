// Matrix products grouped by expert with ragged sizes, and the routed experts' backward pass made of them (formulas: allocmoe.h).
//
//   rows_kernel       y = x W_e^T and dx = dy W_e: a row's products with its group's weight
//   weights_kernel    dW_e = dy^T x: the contraction runs over the group's rows; split_weights_kernel the same for few tiles
//   expert_du_kernel  u = x W13_e^T again, dh = dy W2_e, and from both h, du1 and du3
//
// tcgen05 reads K-major and MN-major operands alike (two bits of the instruction descriptor), so no operand is ever transposed in memory.
// Bound by the tensor cores where a group has some hundred rows, by the weights' bytes (read or written once) where it has few.
//
// Which operand is M: an expert's rows come in any number, its weight does not.  rows_kernel and expert_du_kernel put 128 (a CTA) or
// 256 (a CTA pair, cta_group::2) rows of the WEIGHT on M and the list's rows on N, which the instruction takes in steps of 16 (32): an
// expert of 192 rows costs 192, where rows on M would cost 256 or 384.  The accumulator then holds a column of the output in each lane;
// tcgen05.ld in its 16x256b shape hands out the fragments that stmatrix.trans stores, so a 32 x 32 piece is transposed on
// its way through shared memory by four instructions, and leaves as 64-byte rows.
//
// All three are persistent, one CTA an SM or one CTA pair a TPC.  Warp 0 issues TMA loads into a ring of stages of 64 along the
// contraction, warp 1 the products, eight warps read the finished accumulator while the next tile's products run.
#include <cuda.h>

#include "common.cuh"
#include "tmap.h"
#include "train.h"

namespace allocmoe {

constexpr int kGM = 128;                 // rows of the accumulator in one CTA
constexpr int kGN = 256;                 // columns of an accumulator
constexpr int kGK = 64;                  // contraction of a stage
constexpr int kGThreads = 384;           // loads, products, ragged loads, one idle, eight warps of results
constexpr int kGABytes = kGM * kGK * 2;  // 16 KB
constexpr int kGMostStages = 8;
constexpr int kGMostGroups = 128;
constexpr int kGBoxBytes = 64 * 64 * 2;  // an MN-major box: 64 columns of 64 rows

struct GroupedCtl {
  uint64_t full[kGMostStages], empty[kGMostStages], ragged[kGMostStages];
  uint64_t acc_full[2], acc_empty[2], u_empty, drain;
  uint64_t part_full, part_free;         // partial sums of a cluster
  uint32_t tmem_base;
  volatile int abort_flag;
  volatile uint32_t progress;            // stages that the producer has filled
  int total_tiles;
  int longest;                           // rows of the longest group
  int row_start[kGMostGroups], row_end[kGMostGroups];
  int tile_start[kGMostGroups + 1];
};

// When a launch may touch global memory.  kAfterLast: once everything ahead of it in the stream is complete; it lets its own follower
// start only then.  kBesideLast: at once, for a launch that does not need its predecessor's results but those of a launch before
// that.  The predecessor, kAfterLast or reached through such, has let it start after those were complete; so it takes the SMs that the
// predecessor leaves in its last round of tiles.  Every launch waits for its predecessor before it ends, so whoever waits for the last waits
// for all.
enum class GroupedStart { kAfterLast, kBesideLast };

// What the three kernels share: barriers, TMEM, the table of groups, the way out.
template <bool kPair>
struct GroupedFrame {
  GroupedCtl& ctl;
  int tid, lane, warp, first_tile, tile_step;
  uint32_t rank;                         // of the CTA in its pair; 0 issues the products
  DEV explicit GroupedFrame(GroupedCtl& c)
      : ctl(c), tid(threadIdx.x), lane(threadIdx.x & 31), warp(threadIdx.x >> 5), first_tile(kPair ? blockIdx.x >> 1 : blockIdx.x),
        tile_step(kPair ? gridDim.x >> 1 : gridDim.x), rank(kPair ? cluster_cta_rank() : 0u) {}
  // readers: warps of a CTA that read an accumulator
  DEV void open(int stages, int readers, GroupedStart start) {
    if (tid == 0) {
      for (int s = 0; s < stages; ++s) { mbar_init(&ctl.full[s], kPair ? 2 : 1); mbar_init(&ctl.empty[s], 1); mbar_init(&ctl.ragged[s], 1); }
      for (int a = 0; a < 2; ++a) { mbar_init(&ctl.acc_full[a], 1); mbar_init(&ctl.acc_empty[a], kPair ? 2 * readers : readers); }
      mbar_init(&ctl.u_empty, kPair ? 2 * readers : readers);
      mbar_init(&ctl.drain, 1);
      ctl.abort_flag = 0;
      ctl.progress = 0;
      fence_barrier_init();
    }
    if (warp == 1) {
      if (kPair) { tmem_alloc_pair(&ctl.tmem_base, 512); tmem_relinquish_pair(); }
      else { tmem_alloc(&ctl.tmem_base, 512); tmem_relinquish(); }
    }
    if (start == GroupedStart::kAfterLast) pdl_wait();
    pdl_launch_dependents();
  }
  DEV void ready() {
    tc_fence_before_sync();
    __syncthreads();
    if (kPair) cluster_sync_all();       // both CTAs' barriers are initialised before either signals the other
    tc_fence_after_sync();
  }
  DEV void close() {
    pdl_wait();                          // this launch does not end before the one ahead of it, whenever it started
    tc_fence_before_sync();
    __syncthreads();
    if (kPair) cluster_sync_all();       // neither CTA leaves (or frees TMEM) while its peer may still touch it
    if (warp == 1) {
      __syncwarp();
      tc_fence_after_sync();
      if (kPair) tmem_dealloc_pair(ctl.tmem_base, 512); else tmem_dealloc(ctl.tmem_base, 512);
    }
  }
  DEV uint32_t leader_bar(uint64_t* bar) const { return kPair ? cluster_addr_of(bar, 0) : 0u; }
  DEV void expect(uint64_t* bar, uint32_t cluster_bar, uint32_t bytes) const {
    if (kPair) mbar_expect_tx_cluster(cluster_bar, bytes); else mbar_expect_tx(bar, bytes);
  }
  DEV void arrive_leader(uint64_t* bar) const {
    if (kPair) mbar_arrive_cluster(cluster_addr_of(bar, 0)); else mbar_arrive(bar);
  }
  DEV void load_2d(void* dst, const void* map, uint64_t* bar, uint32_t cluster_bar, int c0, int c1) const {
    if (kPair) tma_load_2d_pair(dst, map, cluster_bar, c0, c1); else tma_load_2d(dst, map, bar, c0, c1);
  }
  DEV void load_3d(void* dst, const void* map, uint64_t* bar, uint32_t cluster_bar, int c0, int c1, int c2) const {
    if (kPair) tma_load_3d_pair(dst, map, cluster_bar, c0, c1, c2); else tma_load_3d(dst, map, bar, c0, c1, c2);
  }
  DEV void umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) const {
    if (kPair) umma_bf16_pair(d, a, b, idesc, acc); else umma_bf16(d, a, b, idesc, acc);
  }
  DEV void commit(uint64_t* bar) const {
    if (kPair) umma_commit_pair(bar, 3); else umma_commit(bar);
  }
  DEV void finish_products() const {     // every product is complete before TMEM is freed
    if (kPair) umma_commit_pair(&ctl.drain, 1); else umma_commit(&ctl.drain);
    mbar_wait_drain(&ctl.drain, 0u);
  }
  // Every load must have landed before the CTA may leave.  The peer's loads complete on the leader's barriers; it learns of them
  // through `empty`.
  DEV void finish_loads(uint32_t it, uint32_t stages) const {
    for (uint32_t q = it > stages ? it - stages : 0u; q < it; ++q)
      mbar_wait_drain(rank == 0 ? &ctl.full[q % stages] : &ctl.empty[q % stages], (q / stages) & 1u);
  }
};

// Segments clamped to [0, P] and to each other, and the tiles of each; without offsets (E 1) the one segment is all rows.  One warp.
template <typename Tiles>
DEV void grouped_table(GroupedCtl& ctl, const int32_t* offsets, int E, int P, int32_t* dev_status, Tiles tiles_of) {
  const int lane = threadIdx.x & 31;
  int carry_row = 0, carry_tile = 0, longest = 0;
  for (int g0 = 0; g0 < E; g0 += 32) {
    const int g = g0 + lane;
    int at = g < E && offsets != nullptr ? clamp_index(offsets[g], 0, P, dev_status) : 0;
    // a running maximum makes the list non-decreasing
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, at, d);
      if (lane >= d) at = max(at, o);
    }
    at = max(at, carry_row);
    const int next = g >= E ? 0 : offsets != nullptr ? max(clamp_index(offsets[g + 1], 0, P, dev_status), at) : P;
    const int tiles = g < E ? tiles_of(next - at) : 0;
    int incl = tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    if (g < E) {
      ctl.row_start[g] = at;
      ctl.row_end[g] = next;
      ctl.tile_start[g] = carry_tile + incl - tiles;
      longest = max(longest, next - at);
    }
    carry_row = __shfl_sync(0xffffffffu, at, 31);
    carry_tile += __shfl_sync(0xffffffffu, incl, 31);
  }
  longest = __reduce_max_sync(0xffffffffu, longest);
  if (lane == 0) {
    ctl.tile_start[E] = carry_tile;
    ctl.total_tiles = carry_tile;
    ctl.longest = longest;
  }
}

// ------------------------------------------------------------------------------------------------ a contraction shared by a cluster
// With few tiles most SMs are idle and a CTA's own loads and products bound the launch.  Then a cluster of CTAs shares each tile: every CTA
// takes a part of the contraction, its eight warps of results leave the accumulators in shared memory as [accumulator][list row][weight row]
// (a lane holds a weight row, so 32 lanes write 128 bytes), and each CTA adds up a share of the tile's (list row, four weight rows) over the
// cluster, in the CTAs' order.  Loads and products of the next tile go on meanwhile.  One group, without and with (us): 200 rows of 4096 -> 1024
// 20.6 and 10.9, 1000 of 4096 -> 512 23.2 and 12.7, 64 of 4096 -> 512 11.8 and 9.2, one of 4096 -> 4096 13.0 and 11.5.
constexpr int kSplitMost = 8;
constexpr int kPartRows = 64;            // list rows of such a tile, at most
DEV float4 ld_cluster_f32x4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
template <int kAccs>
struct PartSums {
  static constexpr size_t kBytes = (size_t)kAccs * kPartRows * kGM * 4;
  GroupedCtl& ctl;
  float* sums;
  int parts, part, lane;
  DEV PartSums(GroupedCtl& c, void* place, int n) : ctl(c), sums(static_cast<float*>(place)), parts(n), part((int)cluster_cta_rank()), lane(threadIdx.x & 31) {}
  // One thread, in front of the frame's open().
  DEV static void init(GroupedCtl& c, int n) {
    mbar_init(&c.part_full, 8 * n);
    mbar_init(&c.part_free, 8 * n);
  }
  // This warp's accumulators of the n-th tile; slots: their TMEM columns.  False: a wait ran out.
  DEV bool write(uint32_t n, int rows, const uint32_t (&slots)[kAccs], volatile int* abort_flag, int32_t* dev_status) {
    const int q = (threadIdx.x >> 5) & 3, half = (int)((threadIdx.x >> 5) - 4) >> 2;
    if (!mbar_spin_bounded_warp(&ctl.part_free, (n & 1u) ^ 1u, abort_flag, dev_status, 2 * kWaitLimitClk)) return false;
    mbar_try_wait_acquire_cluster(&ctl.part_free, (n & 1u) ^ 1u);        // the cluster has read the last tile's sums
    if (half * 32 < rows) {
#pragma unroll
      for (int a = 0; a < kAccs; ++a) {
        uint32_t v[32];
        tmem_ld_32x32(ctl.tmem_base + ((uint32_t)(q * 32) << 16) + slots[a] + half * 32, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; ++i) sums[(a * kPartRows + half * 32 + i) * kGM + q * 32 + lane] = __uint_as_float(v[i]);
      }
    }
    tc_fence_before_sync();
    __syncwarp();
    return true;
  }
  // Behind write(): until every warp of the cluster has written.
  DEV bool publish(uint32_t n, volatile int* abort_flag, int32_t* dev_status) {
    if (lane < parts) mbar_arrive_release_cluster(cluster_addr_of(&ctl.part_full, (uint32_t)lane));
    if (!mbar_spin_bounded_warp(&ctl.part_full, n & 1u, abort_flag, dev_status, 2 * kWaitLimitClk)) return false;
    mbar_try_wait_acquire_cluster(&ctl.part_full, n & 1u);
    return true;
  }
  DEV void joined(int row, int col, float4 (&s)[kAccs]) const {
#pragma unroll
    for (int a = 0; a < kAccs; ++a) s[a] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int k = 0; k < parts; ++k) {
      const uint32_t from = cluster_addr_of(sums + row * kGM + col, (uint32_t)k);
#pragma unroll
      for (int a = 0; a < kAccs; ++a) {
        const float4 v = ld_cluster_f32x4(from + a * kPartRows * kGM * 4);
        s[a] = make_float4(s[a].x + v.x, s[a].y + v.y, s[a].z + v.z, s[a].w + v.w);
      }
    }
  }
  DEV void release() const {             // this warp has read what it needs
    __syncwarp();
    if (lane < parts) mbar_arrive_release_cluster(cluster_addr_of(&ctl.part_free, (uint32_t)lane));
  }
};

// ------------------------------------------------------------------------------------------------ weight rows on M, list rows on N
// A group's rows are cut into equal pieces of at most kMost, each a multiple of kStep but for what the last has left.
template <int kMost, int kStep>
struct RowCut {
  DEV static int pieces(int rows) { return (rows + kMost - 1) / kMost; }
  DEV static int size(int rows) {
    const int n = pieces(rows);
    return ((rows + n - 1) / n + kStep - 1) / kStep * kStep;
  }
};
struct RowTile {
  int e, block;            // group, and block of weight rows
  int row0, valid, n;      // first list row, how many, and their number in the product
};
// Blocks of weight rows outermost, pieces of rows innermost: CTAs that run at the same time share a weight tile through L2.
template <int kMost, int kStep>
struct RowWalk {
  const GroupedCtl& c;
  int g = 0;
  DEV explicit RowWalk(const GroupedCtl& ctl) : c(ctl) {}
  DEV RowTile at(int tile) {             // tile numbers never decrease
    using Cut = RowCut<kMost, kStep>;
    while (tile >= c.tile_start[g + 1]) ++g;
    const int local = tile - c.tile_start[g], lo = c.row_start[g], rows = c.row_end[g] - lo;
    const int pieces = Cut::pieces(rows), size = Cut::size(rows);
    RowTile t;
    t.e = g;
    t.block = local / pieces;
    const int first = local % pieces * size;
    t.row0 = lo + first;
    t.valid = min(size, rows - first);
    t.n = (t.valid + kStep - 1) / kStep * kStep;
    return t;
  }
};

constexpr int kRowMaps = 8;              // boxes of 16, 32 .. 128 list rows
struct RowMaps {
  CUtensorMap m[kRowMaps];
};

// Eight columns of 16 lanes from TMEM four times over: thread t gets lanes t / 4 and t / 4 + 8, columns 8i + 2 (t % 4) and the next.
DEV void tmem_ld_16x256b_x4(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
DEV void stmatrix_x4_trans(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// A piece of 32 list rows x 32 columns (64 bytes a row) in a warp's shared memory; the 16-byte pieces of a row are swapped by its
// number, so that eight rows of one column block lie in different banks.
constexpr int kPieceBytes = 32 * 64;
DEV int piece_at(int row, int chunk) { return row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4); }
// One half (16 columns) of a piece from its fragments: w[2i] columns 0..7, w[2i + 1] columns 8..15 of rows 8i .. 8i+7.
DEV void piece_store_half(unsigned char* buf, int half, int lane, const uint32_t (&w)[8]) {
  const int row = lane & 7, chunk = half * 2 + ((lane >> 3) & 1), block = lane >> 4;
  const uint32_t base = smem_u32(buf);
  stmatrix_x4_trans(base + piece_at(block * 8 + row, chunk), w[0], w[1], w[2], w[3]);
  stmatrix_x4_trans(base + piece_at(16 + block * 8 + row, chunk), w[4], w[5], w[6], w[7]);
}
// The valid rows of a piece to global memory; columns from n_cols on do not exist (n_cols is a multiple of 8).
DEV void piece_copy_out(const unsigned char* buf, uint16_t* out, size_t ld, int row0, int valid, int col0, int n_cols, int lane) {
  const int chunk = lane & 3, col = col0 + chunk * 8;
  if (col >= n_cols) return;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int row = k * 8 + (lane >> 2);
    if (row < valid) *reinterpret_cast<uint4*>(out + (size_t)(row0 + row) * ld + col) = *reinterpret_cast<const uint4*>(buf + piece_at(row, chunk));
  }
}

struct RowsParams {
  const int32_t* offsets;
  int E, P;
  int n_cols;          // columns of the output: rows (kT: columns) of a group's weight
  int k_len;           // length of the contraction
  uint16_t* out;       // [P, n_cols]
  int32_t* dev_status;
  GroupedStart start;
  int parts;           // kSplit: CTAs of a cluster
};

// kPair: 256 weight rows and up to 256 list rows, for many rows a group.  Else 128 weight rows and up to 64 list rows: for few, where
// the weights' bytes decide and more of them are in flight.  64 groups of 2816 x 2048: 192 rows each 157 us (181 at the power cap), 74 % of
// HBM; three rows each 105 us, 7.0 TB/s; the six groups of one token 14.5 us.
template <bool kPair>
struct RowsRing {
  static constexpr int kMost = kPair ? 256 : 64, kStep = kPair ? 32 : 16;
  static constexpr int kBBytes = (kPair ? kMost / 2 : kMost) * kGK * 2, kStageBytes = kGABytes + kBBytes;
  static constexpr int kStages = kPair ? 6 : 8;                       // 192 KB either way
  static constexpr size_t kBytes = (size_t)kStages * kStageBytes;
};

constexpr int kRowsSplitStages = 7;
template <bool kT, bool kPair, bool kSplit>
__global__ void __launch_bounds__(kGThreads, 1)
rows_kernel(const RowsParams p, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ RowMaps maps) {
  using Ring = RowsRing<kPair>;
  using Walk = RowWalk<Ring::kMost, Ring::kStep>;
  static_assert(!(kPair && kSplit), "a cluster is either a pair or shares a contraction");
  constexpr int kTileM = kGM * (kPair ? 2 : 1), kStages = kSplit ? kRowsSplitStages : Ring::kStages;
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
  unsigned char* staging = ring + (size_t)kStages * Ring::kStageBytes;      // kSplit: the partial sums
  GroupedFrame<kPair> f(*reinterpret_cast<GroupedCtl*>(staging + (kSplit ? PartSums<1>::kBytes : 8 * kPieceBytes)));
  GroupedCtl& ctl = f.ctl;
  const int lane = f.lane, warp = f.warp;
  if (f.tid == 0) prefetch_tensormap(&map_w);
  int first_block = 0, k_blocks = (p.k_len + kGK - 1) / kGK;       // of the contraction: all, or this CTA's
  if constexpr (kSplit) {
    const int part = (int)cluster_cta_rank(), all = k_blocks;
    first_block = all * part / p.parts;
    k_blocks = all * (part + 1) / p.parts - first_block;
    f.first_tile = (int)blockIdx.x / p.parts;
    f.tile_step = (int)gridDim.x / p.parts;
    if (f.tid == 0) PartSums<1>::init(ctl, p.parts);
  }
  f.open(kStages, 8, p.start);
  if (warp == 2) {
    const int blocks = (p.n_cols + kTileM - 1) / kTileM;
    grouped_table(ctl, p.offsets, p.E, p.P, p.dev_status, [&](int rows) { return RowCut<Ring::kMost, Ring::kStep>::pieces(rows) * blocks; });
  }
  f.ready();
  if (kSplit) cluster_sync_all();        // every CTA's barriers are initialised before another signals them
  const int total_tiles = ctl.total_tiles;
  volatile int* abort_flag = &ctl.abort_flag;
  Walk walk(ctl);

  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0, s = 0, ph = 0;
      bool ok = true;
      for (int tile = f.first_tile; ok && tile < total_tiles; tile += f.tile_step) {
        const RowTile t = walk.at(tile);
        const int w0 = t.block * kTileM + (int)f.rank * kGM;
        const int rows = kPair ? t.n / 2 : t.n, row0 = t.row0 + (int)f.rank * rows;     // this CTA's part of the list rows
        const CUtensorMap* mb = &maps.m[rows / 16 - 1];
        for (int kb = 0; kb < k_blocks; ++kb) {
          if (!(ok = mbar_wait_bounded(&ctl.empty[s], ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
          unsigned char* sa = ring + s * Ring::kStageBytes;
          uint64_t* bar = &ctl.full[s];
          const uint32_t cbar = f.leader_bar(bar);
          const int k0 = (first_block + kb) * kGK;
          f.expect(bar, cbar, kGABytes + (uint32_t)rows * (kGK * 2));
          if constexpr (kT) {
            f.load_3d(sa, &map_w, bar, cbar, w0, k0, t.e);
            f.load_3d(sa + kGBoxBytes, &map_w, bar, cbar, w0 + 64, k0, t.e);
          } else {
            f.load_3d(sa, &map_w, bar, cbar, k0, w0, t.e);
          }
          f.load_2d(sa + kGABytes, mb, bar, cbar, k0, row0);
          ctl.progress = ++it;
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
      }
      f.finish_loads(it, kStages);
    }
  } else if (warp == 1) {
    if (f.rank == 0 && elect_one()) {
      uint32_t s = 0, ph = 0, n = 0;
      bool ok = true;
      for (int tile = f.first_tile; ok && tile < total_tiles; tile += f.tile_step, ++n) {
        const RowTile t = walk.at(tile);
        const uint32_t idesc = umma_idesc_bf16(kTileM, t.n) | (kT ? 1u << 15 : 0u), a = n & 1u, d = ctl.tmem_base + a * kGN;
        if (!(ok = mbar_wait_bounded(&ctl.acc_empty[a], ((n >> 1) & 1u) ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
        tc_fence_after_sync();
        for (int kb = 0; kb < k_blocks; ++kb) {
          if (!(ok = mbar_wait_bounded(&ctl.full[s], ph, abort_flag, p.dev_status, kWaitLimitClk))) break;
          tc_fence_after_sync();
          const uint32_t sa = smem_u32(ring + s * Ring::kStageBytes);
          const uint64_t da = kT ? umma_desc_mn_sw128(sa, kGBoxBytes) : umma_desc_sw128(sa), db = umma_desc_sw128(sa + kGABytes);
#pragma unroll
          for (int k = 0; k < kGK / 16; ++k) f.umma(d, da + (uint64_t)(k * (kT ? 128 : 2)), db + (uint64_t)(k * 2), idesc, (kb | k) != 0 ? 1u : 0u);
          f.commit(&ctl.empty[s]);
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
        if (ok) f.commit(&ctl.acc_full[a]);
      }
      f.finish_products();
    }
  } else if (kSplit && warp >= 4) {
    PartSums<1> sums(ctl, staging, p.parts);
    const int thread = (warp - 4) * 32 + lane;
    uint32_t n = 0;
    for (int tile = f.first_tile; tile < total_tiles; tile += f.tile_step, ++n) {
      const RowTile t = walk.at(tile);
      const uint32_t a = n & 1u, slots[1] = {a * kGN};
      if (!mbar_spin_progress_warp(&ctl.acc_full[a], (n >> 1) & 1u, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk)) break;
      tc_fence_after_sync();
      if (!sums.write(n, t.n, slots, abort_flag, p.dev_status)) break;
      if (lane == 0) mbar_arrive(&ctl.acc_empty[a]);
      if (!sums.publish(n, abort_flag, p.dev_status)) break;
      const int items = t.valid * (kGM / 4), to = items * (sums.part + 1) / p.parts;
      for (int i = items * sums.part / p.parts + thread; i < to; i += 256) {
        const int row = i / (kGM / 4), c = i % (kGM / 4) * 4, col = t.block * kTileM + c;
        if (col >= p.n_cols) continue;
        float4 s[1];
        sums.joined(row, c, s);
        *reinterpret_cast<uint2*>(p.out + (size_t)(t.row0 + row) * p.n_cols + col) = make_uint2(pack_bf16x2(s[0].x, s[0].y), pack_bf16x2(s[0].z, s[0].w));
      }
      sums.release();
    }
  } else if (warp >= 4) {
    const int q = warp & 3;
    unsigned char* buf = staging + (warp - 4) * kPieceBytes;
    uint32_t n = 0;
    for (int tile = f.first_tile; tile < total_tiles; tile += f.tile_step, ++n) {
      const RowTile t = walk.at(tile);
      const uint32_t a = n & 1u;
      if (!mbar_spin_progress_warp(&ctl.acc_full[a], (n >> 1) & 1u, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk)) break;
      tc_fence_after_sync();
      const uint32_t taddr = ctl.tmem_base + ((uint32_t)(q * 32) << 16) + a * kGN;
      const int col0 = t.block * kTileM + (int)f.rank * kGM + q * 32;
      if (col0 < p.n_cols)
#pragma unroll 1
        for (int r = ((warp - 4) >> 2) * 32; r < t.valid; r += 64) {       // the two warps of a quarter take turns
          uint32_t v[2][16];
          tmem_ld_16x256b_x4(taddr + r, v[0]);
          tmem_ld_16x256b_x4(taddr + (16u << 16) + r, v[1]);
          tmem_ld_wait();
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = pack_bf16x2(__uint_as_float(v[h][2 * i]), __uint_as_float(v[h][2 * i + 1]));
            piece_store_half(buf, h, lane, w);
          }
          __syncwarp();
          piece_copy_out(buf, p.out, (size_t)p.n_cols, t.row0 + r, t.valid - r, col0, p.n_cols, lane);
          __syncwarp();
        }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) f.arrive_leader(&ctl.acc_empty[a]);
    }
  }
  if (kSplit) cluster_sync_all();        // no CTA leaves while another reads its sums
  f.close();
}

// ------------------------------------------------------------------------------------------------ the contraction over the rows
// Ragged ends: the last block of 64 rows may reach into the next segment.  Products are issued for whole groups of 16 rows; where the
// last group is not full, its rows are fetched one by one, as boxes of 32, 16 .. 1 rows by the lanes of warp 2, and the rows missing to 16 as
// boxes that start behind the last row of the tensor, which TMA fills with zeros.  So nothing of another segment enters (a zero in one
// operand alone would not do against a NaN in the other), no thread writes operands, and the stage needs no hand-over between the CTAs
// of a pair: an arrival that releases at cluster scope took 1300 to 2000 clocks of a tile's 5000 under the stores' traffic.
// Into fp32: the tensor core's accumulator truncates, so segments are cut into pieces of 512 rows, added to one another in fp32 in global
// memory, in order: all pieces of a tile belong to one accumulator and one group of warps, whose threads add to what they stored.
// Into bf16: one accumulation up to 32 768 rows.  With terms of one sign it is low by 2e-4 of the sum there, a twentieth of the result's rounding,
// and by 1.6e-3 at 2^18 rows, so longer segments are cut too.  Their running sum takes the second accumulator's place in TMEM, the first group of
// result warps adds a piece to it and the second has nothing to do; that holds for the whole launch where any segment is that long (one group of
// 65 536 rows to 2816 x 2048 665 us, 662 in one accumulation; one of 40 960 beside 63 of 130 rows 680, 630).
// Results: two groups of four warps, one for each accumulator, so that one reads TMEM and packs while the other stores.  bf16 leaves as
// whole lines copied out of shared memory, fp32 by TMA.  Writes alone are bound at 5.5 to 6.2 TB/s with one CTA an SM (7.5 for a plain
// fill).  738 MB of bf16 gradients (64 groups of 2816 x 2048) from three rows a group: 154 us with line copies by eight warps on both
// accumulators, 130 with TMA stores by them, 117 as it is; from 192 rows a group 187 us, 142 GFLOP, shared memory 74 % busy.
// The same in fp32 from 12 288 rows (64 groups of 2048 x 1408): 171 us.
template <bool kPair, bool kF32>
struct WeightsRing {
  static constexpr int kBBytes = kGN * kGK * 2 / (kPair ? 2 : 1), kStageBytes = kGABytes + kBBytes;
  static constexpr int kStages = (kPair ? 6 : 4) - (kF32 ? 1 : 0);
  static constexpr size_t kBytes = (size_t)kStages * kStageBytes;
  static constexpr int kStageOut = kF32 ? 8192 : 4096;                 // a warp's staging: boxes of 32 rows of 128 bytes, two for fp32
};
constexpr int kGPieceLog2 = 9;           // rows that one accumulation into fp32 takes: 512
constexpr int kGLongLog2 = 15;           // the same into bf16: 32 768
constexpr int kGHeights = 7;             // boxes of 1, 2 .. 64 rows

struct WeightsProblem {
  int m_rows, n_cols;  // the output of a group
  void* out;           // [E, m_rows, n_cols]
};
// One or two products over the same segments: the second's tiles follow the first's.
struct WeightsParams {
  const int32_t* offsets;
  int E, P;
  int problems;
  WeightsProblem q[2];
  bool add;            // fp32: add to what the output holds
  int32_t* dev_status;
  GroupedStart start;
};
struct WeightsMaps {
  CUtensorMap a[kGHeights], b[kGHeights];
  CUtensorMap out;     // fp32
};
struct WeightsMaps2 {
  WeightsMaps q[2];
};
struct WeightsTile {
  int q, e, m0, n0, k0, k_end;
  int pieces;
};
// Tiles of a group: column blocks innermost.  The walk goes on by a fixed step, taken apart once for each problem.
template <int kTileM, int kPieceLog2>
struct WeightsWalk {
  const GroupedCtl& c;
  int step, q = 0, n_blocks, m_blocks, g = 0, mb, nb, step_m, step_n;
  DEV WeightsWalk(const GroupedCtl& ctl, const WeightsParams& p, int first, int s) : c(ctl), step(s) { enter(p, first); }
  DEV void enter(const WeightsParams& p, int tile) {           // the tile-th one of problem q
    n_blocks = (p.q[q].n_cols + kGN - 1) / kGN;
    m_blocks = (p.q[q].m_rows + kTileM - 1) / kTileM;
    g = 0;
    mb = tile / n_blocks;
    nb = tile - mb * n_blocks;
    step_m = step / n_blocks;
    step_n = step - step_m * n_blocks;
  }
  DEV bool at(const WeightsParams& p, WeightsTile& t) {        // false: no tile is left
    while (true) {
      while (mb >= m_blocks) { mb -= m_blocks; ++g; }
      if (g < p.E) break;
      if (q + 1 >= p.problems) return false;
      const int left = ((g - p.E) * m_blocks + mb) * n_blocks + nb;
      ++q;
      enter(p, left);
    }
    t.q = q;
    t.e = g;
    t.m0 = mb * kTileM;
    t.n0 = nb * kGN;
    t.k0 = c.row_start[g];
    t.k_end = c.row_end[g];
    t.pieces = max(1, (t.k_end - t.k0 + (1 << kPieceLog2) - 1) >> kPieceLog2);
    mb += step_m;
    nb += step_n;
    if (nb >= n_blocks) { nb -= n_blocks; ++mb; }
    return true;
  }
};
template <int kPieceLog2>
struct WeightsRun {
  int k0, blocks, last;    // first row, blocks of 64, rows in the last block
  DEV WeightsRun(const WeightsTile& t, int piece) {
    k0 = t.k0 + (piece << kPieceLog2);
    const int rows = min(1 << kPieceLog2, t.k_end - k0);
    blocks = (rows + kGK - 1) / kGK;
    last = rows - (blocks - 1) * kGK;
  }
};

template <bool kPair, bool kF32>
__global__ void __launch_bounds__(kGThreads, 1)
weights_kernel(const __grid_constant__ WeightsParams p, const __grid_constant__ WeightsMaps2 maps2) {
  using Ring = WeightsRing<kPair, kF32>;
  constexpr int kTileM = kGM * (kPair ? 2 : 1), kStages = Ring::kStages, kStageBytes = Ring::kStageBytes, kBoxes = kStageBytes / kGBoxBytes;
  constexpr int kPieceLog2 = kF32 ? kGPieceLog2 : kGLongLog2;
  using Run = WeightsRun<kPieceLog2>;
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
  unsigned char* staging = ring + Ring::kBytes;
  GroupedFrame<kPair> f(*reinterpret_cast<GroupedCtl*>(staging + 8 * Ring::kStageOut));
  GroupedCtl& ctl = f.ctl;
  const int lane = f.lane, warp = f.warp;
  if (f.tid == 0) {
    prefetch_tensormap(&maps2.q[0].a[kGHeights - 1]);
    prefetch_tensormap(&maps2.q[0].b[kGHeights - 1]);
  }
  f.open(kStages, 4, p.start);
  if (warp == 2) grouped_table(ctl, p.offsets, p.E, p.P, p.dev_status, [](int) { return 0; });
  f.ready();
  volatile int* abort_flag = &ctl.abort_flag;
  WeightsWalk<kTileM, kPieceLog2> walk(ctl, p, f.first_tile, f.tile_step);
  WeightsTile t;
  const bool one_place = !kF32 && ctl.longest > 1 << kPieceLog2;       // one accumulator, its running sum in the other's place

  if (warp == 0) {
    // ======================= loads of whole blocks (each CTA its own part) =======================
    if (elect_one()) {
      uint32_t it = 0, s = 0, ph = 0;
      bool ok = true;
      while (ok && walk.at(p, t)) {
        const WeightsMaps& maps = maps2.q[t.q];
        const int m0 = t.m0 + (int)f.rank * kGM, n0 = t.n0 + (int)f.rank * (kGN / 2);
        for (int piece = 0; ok && piece < t.pieces; ++piece) {
          const Run run(t, piece);
          for (int kb = 0; kb < run.blocks; ++kb) {
            if (!(ok = mbar_wait_bounded(&ctl.empty[s], ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
            if (kb == run.blocks - 1 && (run.last & 15) != 0) {
              mbar_arrive(&ctl.ragged[s]);           // the stage is free: warp 2 fills it
            } else {
              unsigned char* stage = ring + s * kStageBytes;
              uint64_t* bar = &ctl.full[s];
              const uint32_t cbar = f.leader_bar(bar);
              const int row = run.k0 + kb * kGK;
              f.expect(bar, cbar, kStageBytes);
#pragma unroll
              for (int j = 0; j < 2; ++j) f.load_2d(stage + j * kGBoxBytes, &maps.a[kGHeights - 1], bar, cbar, m0 + j * 64, row);
#pragma unroll
              for (int j = 0; j < kBoxes - 2; ++j) f.load_2d(stage + (2 + j) * kGBoxBytes, &maps.b[kGHeights - 1], bar, cbar, n0 + j * 64, row);
            }
            ctl.progress = ++it;
            if (++s == kStages) { s = 0; ph ^= 1u; }
          }
        }
      }
      f.finish_loads(it, kStages);
    }
  } else if (warp == 1) {
    // ======================= products (the leader alone) =======================
    if (f.rank == 0 && elect_one()) {
      constexpr uint32_t idesc = umma_idesc_bf16(kTileM, kGN) | 1u << 15 | 1u << 16;     // both operands MN-major
      uint32_t s = 0, ph = 0, a = 1, uses[2] = {0, 0};
      bool ok = true;
      while (ok && walk.at(p, t)) {
        a = one_place ? 0u : a ^ 1u;
        for (int piece = 0; ok && piece < t.pieces; ++piece) {
          const Run run(t, piece);
          const uint32_t d = ctl.tmem_base + a * kGN, n = a == 0 ? uses[0]++ : uses[1]++;
          if (!(ok = mbar_wait_bounded(&ctl.acc_empty[a], (n & 1u) ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
          tc_fence_after_sync();
          for (int kb = 0; kb < run.blocks; ++kb) {
            const int rows = kb == run.blocks - 1 ? run.last : kGK;
            if (!(ok = mbar_wait_bounded(&ctl.full[s], ph, abort_flag, p.dev_status, kWaitLimitClk))) break;
            tc_fence_after_sync();
            const uint32_t sa = smem_u32(ring + s * kStageBytes);
            const uint64_t da = umma_desc_mn_sw128(sa, kGBoxBytes), db = umma_desc_mn_sw128(sa + kGABytes, kGBoxBytes);
            if (rows < kGK) {
              for (int k = 0; k * 16 < rows; ++k) f.umma(d, da + (uint64_t)(k * 128), db + (uint64_t)(k * 128), idesc, (kb | k) != 0 ? 1u : 0u);
            } else {
#pragma unroll
              for (int k = 0; k < kGK / 16; ++k) f.umma(d, da + (uint64_t)(k * 128), db + (uint64_t)(k * 128), idesc, (kb | k) != 0 ? 1u : 0u);
            }
            f.commit(&ctl.empty[s]);
            if (++s == kStages) { s = 0; ph ^= 1u; }
          }
          if (ok) f.commit(&ctl.acc_full[a]);
        }
      }
      f.finish_products();
    }
  } else if (warp == 2) {
    // ======================= loads of a last block whose last group of 16 rows is not full (each CTA its own part) =======================
    uint32_t it = 0, used = 0;                   // used: a bit a stage, the parity of `ragged`
    bool ok = true;
    while (ok && walk.at(p, t)) {
      const WeightsMaps& maps = maps2.q[t.q];
      const int m0 = t.m0 + (int)f.rank * kGM, n0 = t.n0 + (int)f.rank * (kGN / 2);
      for (int piece = 0; piece < t.pieces; ++piece) {
        const Run run(t, piece);
        it += run.blocks;
        if (run.blocks == 0 || (run.last & 15) == 0) continue;
        // Not `empty`: a wait by parity must not be a phase ahead, and this warp passes over the stages in between.  `ragged` of a stage
        // goes on once for each of its ragged blocks, and not again before this warp has filled the stage.
        const uint32_t s = (it - 1) % kStages;
        if (!(ok = mbar_spin_progress_warp(&ctl.ragged[s], used >> s & 1u, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk))) break;
        used ^= 1u << s;
        unsigned char* stage = ring + s * kStageBytes;
        uint64_t* bar = &ctl.full[s];
        const uint32_t cbar = f.leader_bar(bar);
        const int row = run.k0 + (run.blocks - 1) * kGK, none = 16 - (run.last & 15);
        if (lane == 0) f.expect(bar, cbar, (uint32_t)(run.last + none) * 128u * kBoxes);
        __syncwarp();
        for (int i = lane; i < 10 * kBoxes; i += 32) {
          const int slot = i / kBoxes, j = i - slot * kBoxes;
          const int bit = slot < 6 ? 5 - slot : 9 - slot, count = slot < 6 ? run.last : none;      // rows of the segment, then the missing ones
          if (count >> bit & 1) {
            const int before = count >> (bit + 1) << (bit + 1);            // rows in the boxes of the higher bits
            f.load_2d(stage + j * kGBoxBytes + ((slot < 6 ? 0 : run.last) + before) * 128, j < 2 ? &maps.a[bit] : &maps.b[bit], bar, cbar,
                      j < 2 ? m0 + j * 64 : n0 + (j - 2) * 64, slot < 6 ? row + before : p.P);
          }
        }
        __syncwarp();
      }
    }
  } else if (warp >= 4) {
    // ======================= results =======================
    const int quarter = warp & 3, group = (warp - 4) >> 2;
    unsigned char* buf = staging + (warp - 4) * Ring::kStageOut;
    const bool issuer = elect_one();
    uint32_t n = 0, turn = 1, box = 0;
    bool ok = true;
    while (ok && walk.at(p, t)) {
      turn ^= 1u;
      if ((one_place ? 0u : turn) != (uint32_t)group) continue;
      const int row0 = t.m0 + (int)f.rank * kGM + quarter * 32, m_rows = p.q[t.q].m_rows, n_total = p.q[t.q].n_cols;
      const WeightsMaps& maps = maps2.q[t.q];
      const bool none = t.k_end == t.k0;
      for (int piece = 0; piece < t.pieces; ++piece, ++n) {
        if (!(ok = mbar_spin_progress_warp(&ctl.acc_full[group], n & 1u, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk))) break;
        tc_fence_after_sync();
        const bool add = kF32 && (p.add || piece > 0);
        const int n_cols = row0 < m_rows && !(none && add) ? min(kGN, n_total - t.n0) : 0;
        const uint32_t taddr = ctl.tmem_base + ((uint32_t)(quarter * 32) << 16) + group * kGN;
        // an addition comes behind what this thread has stored before
        if (kF32 && piece > 0 && issuer) bulk_wait_all();
#pragma unroll 1
        for (int c = 0; c < kGN; c += 64) {
          uint32_t v[64];
          tmem_ld_32x32(taddr + c, *reinterpret_cast<uint32_t(*)[32]>(v));
          tmem_ld_32x32(taddr + c + 32, *reinterpret_cast<uint32_t(*)[32]>(v + 32));
          tmem_ld_wait();
          if (c + 64 >= kGN) {                   // everything is in registers: the accumulator is free
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) f.arrive_leader(&ctl.acc_empty[group]);
          }
          if (c >= n_cols) continue;
          if (none) {
#pragma unroll
            for (int i = 0; i < 64; ++i) v[i] = 0u;
          }
          const int j = lane & 7, r0 = lane >> 3;
          if constexpr (kF32) {
#pragma unroll
            for (int part = 0; part < 2; ++part) {
              if (c + part * 32 >= n_cols) continue;
              unsigned char* mine = buf + (box++ & 1u) * 4096;
              if (issuer) bulk_wait_read<1>();   // the store before last has left this box
              __syncwarp();
#pragma unroll
              for (int i = 0; i < 8; ++i)
                *reinterpret_cast<uint4*>(mine + lane * 128 + ((i ^ j) << 4)) = *reinterpret_cast<const uint4*>(v + part * 32 + 4 * i);
              fence_proxy_async_smem();
              __syncwarp();
              if (issuer) {
                if (add) tma_add_3d(mine, &maps.out, t.n0 + c + part * 32, row0, t.e);
                else tma_store_3d(mine, &maps.out, t.n0 + c + part * 32, row0, t.e);
                bulk_commit();
              }
            }
          } else {
            if (t.pieces > 1) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                uint32_t(&w)[32] = *reinterpret_cast<uint32_t(*)[32]>(v + 32 * h);
                if (piece > 0) {
                  uint32_t sum[32];
                  tmem_ld_32x32(taddr + kGN + c + 32 * h, sum);
                  tmem_ld_wait();
#pragma unroll
                  for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(__uint_as_float(w[i]) + __uint_as_float(sum[i]));
                }
                if (piece + 1 < t.pieces) tmem_st_32x32(taddr + kGN + c + 32 * h, w);
              }
              if (piece + 1 < t.pieces) {
                tmem_st_wait();
                continue;
              }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t* u = v + 8 * i;
              *reinterpret_cast<uint4*>(buf + lane * 128 + ((i ^ j) << 4)) =
                  make_uint4(pack_bf16x2(__uint_as_float(u[0]), __uint_as_float(u[1])), pack_bf16x2(__uint_as_float(u[2]), __uint_as_float(u[3])),
                             pack_bf16x2(__uint_as_float(u[4]), __uint_as_float(u[5])), pack_bf16x2(__uint_as_float(u[6]), __uint_as_float(u[7])));
            }
            __syncwarp();
            uint4 w[8];                          // eight lanes a row of 64 columns, four rows at a time
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = *reinterpret_cast<const uint4*>(buf + (k * 4 + r0) * 128 + ((j ^ ((k * 4 + r0) & 7)) << 4));
            __syncwarp();
            uint16_t* out = static_cast<uint16_t*>(p.q[t.q].out) + ((size_t)t.e * m_rows + row0 + r0) * n_total + t.n0 + c + j * 8;
            const size_t step = 4 * (size_t)n_total;
#pragma unroll
            for (int k = 0; k < 8; ++k, out += step)
              if (row0 + k * 4 + r0 < m_rows && c + j * 8 < n_cols) *reinterpret_cast<uint4*>(out) = w[k];
          }
        }
      }
    }
    if (kF32 && issuer) bulk_wait_all();
  }
  f.close();
}

// ------------------------------------------------------------------------------------------------ few tiles, many rows: the contraction split
// One group or a few with small weights leave most SMs idle above, and what an SM can load bounds the rest (62 to 75 GB/s).  Here a cluster of
// up to 8 CTAs shares a tile of 128 x 64, 128 or 256, each with its part of the rows.  Its eight warps of results hold a running sum of
// 128 columns a thread (pieces of 512 rows), leave it in shared memory behind the last product, and every
// CTA adds its share of the tile's rows over the cluster, in the CTAs' order.  12 153 rows to 232 x 152: 15.6 us (above 85, into fp32 136);
// 16 384 to 64 x 64: 13.8 (77); 12 288 to 64 x 2048, 8.1 us of HBM: 20 (70, 130 into fp32).
struct SplitParams {
  const int32_t* offsets;
  int E, P, m_rows, n_cols, parts;       // parts: CTAs of a cluster
  int m_blocks, n_blocks, tile_n;        // tiles of 128 x tile_n
  bool add;
  void* out;           // [E, m_rows, n_cols]
  int32_t* dev_status;
};
struct SplitMaps {
  CUtensorMap a[kGHeights], b[kGHeights];
};
constexpr int kSplitPiece = (1 << kGPieceLog2) / kGK;      // blocks of 64 rows of one accumulation
constexpr size_t kSplitRing = 4 * 6 * kGBoxBytes;          // four stages of 64 x (128 + 256), more where the tile is smaller
static_assert(kSplitRing >= (size_t)kGM * kGN * 4, "the sums take the ring's place");

template <bool kF32>
__global__ void __launch_bounds__(kGThreads, 1)
split_weights_kernel(const __grid_constant__ SplitParams p, const __grid_constant__ SplitMaps maps) {
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
  GroupedFrame<false> f(*reinterpret_cast<GroupedCtl*>(ring + kSplitRing));
  GroupedCtl& ctl = f.ctl;
  const int lane = f.lane, warp = f.warp, rank = (int)cluster_cta_rank();
  const int tile = blockIdx.x / p.parts, per_group = p.m_blocks * p.n_blocks, e = tile / per_group, in_group = tile - e * per_group;
  const int mb = in_group / p.n_blocks, m0 = mb * kGM, n0 = (in_group - mb * p.n_blocks) * p.tile_n, cols = min(p.tile_n, p.n_cols - n0);
  const int m_boxes = min(2, (p.m_rows - m0 + 63) / 64), n_boxes = (cols + 63) / 64, boxes = m_boxes + n_boxes;
  const int stage_bytes = boxes * kGBoxBytes, stages = min(kGMostStages, (int)kSplitRing / stage_bytes);
  if (f.tid == 0) {
    prefetch_tensormap(&maps.a[kGHeights - 1]);
    prefetch_tensormap(&maps.b[kGHeights - 1]);
  }
  f.open(stages, 8, GroupedStart::kAfterLast);
  if (warp == 2) grouped_table(ctl, p.offsets, p.E, p.P, p.dev_status, [](int) { return 0; });
  f.ready();
  volatile int* abort_flag = &ctl.abort_flag;
  // this CTA's blocks of 64 rows
  const int first_row = ctl.row_start[e], end = ctl.row_end[e], all = (end - first_row + kGK - 1) / kGK;
  const int b0 = (int)((long long)all * rank / p.parts), blocks = (int)((long long)all * (rank + 1) / p.parts) - b0;
  const int k0 = first_row + b0 * kGK, pieces = (blocks + kSplitPiece - 1) / kSplitPiece;

  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0, s = 0, ph = 0;
      for (int b = 0; b < blocks; ++b) {
        if (!mbar_wait_bounded(&ctl.empty[s], ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk)) break;
        unsigned char* stage = ring + s * stage_bytes;
        uint64_t* bar = &ctl.full[s];
        const int row = k0 + b * kGK, rows = min(kGK, end - row);
        if ((rows & 15) == 0) {
          mbar_expect_tx(bar, (uint32_t)stage_bytes);
          for (int j = 0; j < m_boxes; ++j) tma_load_2d(stage + j * kGBoxBytes, &maps.a[kGHeights - 1], bar, m0 + j * 64, row);
          for (int j = 0; j < n_boxes; ++j) tma_load_2d(stage + (m_boxes + j) * kGBoxBytes, &maps.b[kGHeights - 1], bar, n0 + j * 64, row);
        } else {                                 // boxes of 32 .. 1 rows, then of rows behind the tensor's end
          const int none = 16 - (rows & 15);
          mbar_expect_tx(bar, (uint32_t)(rows + none) * 128u * boxes);
          for (int slot = 0; slot < 10; ++slot) {
            const int bit = slot < 6 ? 5 - slot : 9 - slot, count = slot < 6 ? rows : none;
            if (!(count >> bit & 1)) continue;
            const int before = count >> (bit + 1) << (bit + 1), at = ((slot < 6 ? 0 : rows) + before) * 128, from = slot < 6 ? row + before : p.P;
            for (int j = 0; j < m_boxes; ++j) tma_load_2d(stage + j * kGBoxBytes + at, &maps.a[bit], bar, m0 + j * 64, from);
            for (int j = 0; j < n_boxes; ++j) tma_load_2d(stage + (m_boxes + j) * kGBoxBytes + at, &maps.b[bit], bar, n0 + j * 64, from);
          }
        }
        ctl.progress = ++it;
        if (++s == (uint32_t)stages) { s = 0; ph ^= 1u; }
      }
      f.finish_loads(it, (uint32_t)stages);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      const uint32_t idesc = umma_idesc_bf16(kGM, n_boxes * 64) | 1u << 15 | 1u << 16;     // both operands MN-major
      uint32_t s = 0, ph = 0;
      bool ok = true;
      for (int piece = 0; ok && piece < pieces; ++piece) {
        const uint32_t a = piece & 1, d = ctl.tmem_base + a * kGN;
        if (!(ok = mbar_wait_bounded(&ctl.acc_empty[a], (piece >> 1 & 1) ^ 1, abort_flag, p.dev_status, kWaitLimitClk))) break;
        tc_fence_after_sync();
        const int from = piece * kSplitPiece, to = min(blocks, from + kSplitPiece);
        for (int b = from; b < to; ++b) {
          if (!(ok = mbar_wait_bounded(&ctl.full[s], ph, abort_flag, p.dev_status, kWaitLimitClk))) break;
          tc_fence_after_sync();
          const uint32_t sa = smem_u32(ring + s * stage_bytes);
          const uint64_t da = umma_desc_mn_sw128(sa, kGBoxBytes), db = umma_desc_mn_sw128(sa + m_boxes * kGBoxBytes, kGBoxBytes);
          const int rows = min(kGK, end - (k0 + b * kGK));
          for (int k = 0; k * 16 < rows; ++k)
            umma_bf16(d, da + (uint64_t)(k * 128), db + (uint64_t)(k * 128), idesc, (b - from) != 0 || k != 0 ? 1u : 0u);
          umma_commit(&ctl.empty[s]);
          if (++s == (uint32_t)stages) { s = 0; ph ^= 1u; }
        }
        if (ok) umma_commit(&ctl.acc_full[a]);
      }
      f.finish_products();
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, half = (warp - 4) >> 2, width = n_boxes * 64 - half * 128;      // columns that exist behind this warp's first
    float sum[128];
#pragma unroll
    for (int i = 0; i < 128; ++i) sum[i] = 0.f;
    bool ok = true;
#pragma unroll 1
    for (int piece = 0; piece < pieces; ++piece) {
      const uint32_t a = piece & 1;
      if (!(ok = mbar_spin_progress_warp(&ctl.acc_full[a], piece >> 1 & 1, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk))) break;
      tc_fence_after_sync();
      const uint32_t taddr = ctl.tmem_base + ((uint32_t)(quarter * 32) << 16) + a * kGN + half * 128;
#pragma unroll
      for (int c = 0; c < 128; c += 32) {
        if (c >= width) continue;
        uint32_t v[32];
        tmem_ld_32x32(taddr + c, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; ++i) sum[c + i] += __uint_as_float(v[i]);
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.acc_empty[a]);
    }
    // The last product has read its stage: the ring is free.  A row's 16-byte pieces lie in another order in each row of 32.
    if (ok) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i * 4 < width)
          *reinterpret_cast<float4*>(ring + (quarter * 32 + lane) * 1024 + (((half * 32 + i) ^ lane) << 4)) =
              make_float4(sum[4 * i], sum[4 * i + 1], sum[4 * i + 2], sum[4 * i + 3]);
    }
  }
  __syncthreads();
  cluster_sync_all();
  const int rows = kGM / p.parts;
  if (!(p.add && end == first_row))
    for (int i = f.tid; i < rows * (kGN / 4); i += kGThreads) {
      const int r = rank * rows + i / (kGN / 4), c = i % (kGN / 4);
      if (m0 + r >= p.m_rows || c * 4 >= cols) continue;
      const unsigned char* place = ring + r * 1024 + ((c ^ (r & 31)) << 4);
      float4 v[kSplitMost];
#pragma unroll
      for (int k = 0; k < kSplitMost; ++k)
        if (k < p.parts)
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(v[k].x), "=f"(v[k].y), "=f"(v[k].z), "=f"(v[k].w)
                       : "r"(cluster_addr_of(place, (uint32_t)k)));
      float4 a = v[0];
#pragma unroll
      for (int k = 1; k < kSplitMost; ++k)
        if (k < p.parts) a = make_float4(a.x + v[k].x, a.y + v[k].y, a.z + v[k].z, a.w + v[k].w);
      const size_t at = ((size_t)e * p.m_rows + m0 + r) * p.n_cols + n0 + c * 4;
      if constexpr (kF32) {
        float4* out = reinterpret_cast<float4*>(static_cast<float*>(p.out) + at);
        if (p.add) {
          const float4 o = *out;
          a = make_float4(o.x + a.x, o.y + a.y, o.z + a.z, o.w + a.w);
        }
        *out = a;
      } else {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
      }
    }
  cluster_sync_all();                    // no CTA leaves while another reads its sums
  f.close();
}

// ------------------------------------------------------------------------------------------------ experts: u, dh, and what follows from both
// A tile is 128 (a pair: 256) hidden units of an expert times up to 64 (128) of its rows, with three accumulators: dh (W2_e's columns,
// MN-major, against dy), then u1 and u3 (rows of W1 and W3 against x, each block of x loaded once for both).  dh has two places that take
// turns, so the products of the next tile's dh run while this tile's three accumulators are read: 4 x 128 columns of TMEM.  Nothing
// of u or dh touches memory.  64 experts of 2048 x 1408: three rows each 149 us, 7.4 TB/s of weights; 192 rows each 303 us, 10.5 TB/s from L2
// to the SMs (the weights go there once for each 128 rows).
// kSplit, for few tiles: a cluster of up to 8 CTAs shares a tile's contraction and joins the three sums over shared memory (12 experts of
// 3264 x 64 and 129 pairs 35.8 us for the whole backward pass, 58 without; 3 pairs of 3648 x 512 70, 93 without).
struct DuParams {
  const int32_t* offsets;
  int E, P, H, I;
  int subs;            // S sub-experts a group, whose results are summed: routed 1, the shared experts one group of S
  uint16_t* h;         // [P, S*I]
  uint16_t* du;        // [P, S*2I], u1 and u3 of a sub-expert side by side
  int32_t* dev_status;
  GroupedStart start;  // kBesideLast: the launch ahead gathers x
  int parts;           // kSplit: CTAs of a cluster, which share a tile's contraction
};
template <bool kPair>
struct DuRing {
  static constexpr int kMost = kPair ? 128 : 64, kStep = kPair ? 32 : 16;
  static constexpr int kBBytes = 64 * kGK * 2, kStageBytes = kGABytes + kBBytes;      // 24 KB: weight rows and 64 list rows
  static constexpr int kStages = 7;
  static constexpr size_t kBytes = (size_t)kStages * kStageBytes;
};
constexpr int kDuSlot = 128;             // TMEM columns of an accumulator
constexpr int kDuSplitStages = 5;
// h, du1 and du3 of a hidden unit; h as in the forward pass
DEV void expert_unit(float a, float b, float dh, float* vh, float* v1, float* v3) {
  const float den = 1.f + __expf(-a), sg = __fdividef(1.f, den);
  *vh = __fdividef(a * b, den);
  *v3 = dh * (a * sg);
  *v1 = dh * b * (sg * (1.f + a * (1.f - sg)));
}

// The list's rows of x, a warp a row.  Its follower may start once everything ahead of this launch is complete.
__global__ void __launch_bounds__(256)
list_rows_kernel(const uint4* __restrict__ x, const int32_t* __restrict__ perm_token, int T, int row_vec, int rows, uint4* __restrict__ out,
                 int32_t* dev_status) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  for (int p = blockIdx.x * 8 + (threadIdx.x >> 5); p < rows; p += gridDim.x * 8) {
    const uint4* src = x + (size_t)clamp_index(__ldg(perm_token + p), 0, T - 1, dev_status) * row_vec;
    uint4* dst = out + (size_t)p * row_vec;
    for (int c = lane; c < row_vec; c += 128) {
      uint4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + 32 * k < row_vec) v[k] = __ldg(src + c + 32 * k);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + 32 * k < row_vec) dst[c + 32 * k] = v[k];
    }
  }
}

template <bool kPair, bool kSplit>
__global__ void __launch_bounds__(kGThreads, 1)
expert_du_kernel(const DuParams p, const __grid_constant__ CUtensorMap map_w13, const __grid_constant__ CUtensorMap map_w2,
                 const __grid_constant__ RowMaps maps_x, const __grid_constant__ RowMaps maps_dy) {
  static_assert(!(kPair && kSplit), "a cluster is either a pair or shares a contraction");
  using Ring = DuRing<kPair>;
  constexpr int kTileM = kGM * (kPair ? 2 : 1), kStages = kSplit ? kDuSplitStages : Ring::kStages, kStageBytes = Ring::kStageBytes;
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
  unsigned char* staging = ring + (size_t)kStages * kStageBytes;         // kSplit: the partial sums
  GroupedFrame<kPair> f(*reinterpret_cast<GroupedCtl*>(staging + (kSplit ? PartSums<3>::kBytes : 8 * 3 * kPieceBytes)));
  GroupedCtl& ctl = f.ctl;
  const int lane = f.lane, warp = f.warp;
  int first_block = 0, k_blocks = p.H / kGK;     // of the contraction: all, or this CTA's
  if constexpr (kSplit) {
    const int part = (int)cluster_cta_rank(), all = k_blocks;
    first_block = all * part / p.parts;
    k_blocks = all * (part + 1) / p.parts - first_block;
    f.first_tile = (int)blockIdx.x / p.parts;
    f.tile_step = (int)gridDim.x / p.parts;
    if (f.tid == 0) PartSums<3>::init(ctl, p.parts);
  }
  if (f.tid == 0) {
    prefetch_tensormap(&map_w13);
    prefetch_tensormap(&map_w2);
  }
  f.open(kStages, 8, p.start);
  const int sub_blocks = (p.I + kTileM - 1) / kTileM;
  if (warp == 2) {
    const int blocks = sub_blocks * p.subs;
    grouped_table(ctl, p.offsets, p.E, p.P, p.dev_status, [&](int rows) { return RowCut<Ring::kMost, Ring::kStep>::pieces(rows) * blocks; });
  }
  f.ready();
  if (kSplit) cluster_sync_all();        // every CTA's barriers are initialised before another signals them
  const int total_tiles = ctl.total_tiles;
  volatile int* abort_flag = &ctl.abort_flag;
  RowWalk<Ring::kMost, Ring::kStep> walk(ctl);

  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0, s = 0, ph = 0;
      bool ok = true;
      for (int tile = f.first_tile; ok && tile < total_tiles; tile += f.tile_step) {
        const RowTile t = walk.at(tile);
        const int sub = t.block / sub_blocks, matrix = t.e * p.subs + sub, w0 = (t.block - sub * sub_blocks) * kTileM + (int)f.rank * kGM;
        const int rows = kPair ? t.n / 2 : t.n, row0 = t.row0 + (int)f.rank * rows;
        // dh: a stage a block, W2's columns and dy.  u: two stages a block, W1's rows and x, then W3's rows alone.
        for (int step = 0; step < 3 * k_blocks; ++step) {
          if (!(ok = mbar_wait_bounded(&ctl.empty[s], ph ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
          unsigned char* sa = ring + s * kStageBytes;
          uint64_t* bar = &ctl.full[s];
          const uint32_t cbar = f.leader_bar(bar);
          if (step == k_blocks && it == (uint32_t)k_blocks) {          // the first block of x
            pdl_wait();
            fence_proxy_async_global();
          }
          const bool dh = step < k_blocks, up = !dh && ((step - k_blocks) & 1) != 0;
          const int k0 = (first_block + (dh ? step : (step - k_blocks) >> 1)) * kGK;
          f.expect(bar, cbar, kGABytes + (up ? 0u : (uint32_t)rows * (kGK * 2)));
          if (dh) {
            f.load_3d(sa, &map_w2, bar, cbar, w0, k0, matrix);
            f.load_3d(sa + kGBoxBytes, &map_w2, bar, cbar, w0 + 64, k0, matrix);
          } else {
            f.load_3d(sa, &map_w13, bar, cbar, k0, w0, matrix * 2 + (up ? 1 : 0));
          }
          if (!up) f.load_2d(sa + kGABytes, dh ? &maps_dy.m[rows / 16 - 1] : &maps_x.m[rows / 16 - 1], bar, cbar, k0, row0);
          ctl.progress = ++it;
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
      }
      f.finish_loads(it, kStages);
    }
  } else if (warp == 1) {
    if (f.rank == 0 && elect_one()) {
      uint32_t s = 0, ph = 0, n = 0;
      bool ok = true;
      for (int tile = f.first_tile; ok && tile < total_tiles; tile += f.tile_step, ++n) {
        const RowTile t = walk.at(tile);
        const uint32_t idesc = umma_idesc_bf16(kTileM, t.n), tm = ctl.tmem_base;
        if (!(ok = mbar_wait_bounded(&ctl.acc_empty[n & 1u], ((n >> 1) & 1u) ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
        tc_fence_after_sync();
        uint32_t x_stage = 0;                  // where the block of x lies that W3's rows meet too
        for (int step = 0; step < 3 * k_blocks; ++step) {
          if (step == k_blocks) {
            if (!(ok = mbar_wait_bounded(&ctl.u_empty, (n & 1u) ^ 1u, abort_flag, p.dev_status, kWaitLimitClk))) break;
            tc_fence_after_sync();
          }
          if (!(ok = mbar_wait_bounded(&ctl.full[s], ph, abort_flag, p.dev_status, kWaitLimitClk))) break;
          tc_fence_after_sync();
          const bool dh = step < k_blocks, up = !dh && ((step - k_blocks) & 1) != 0;
          const uint32_t sa = smem_u32(ring + s * kStageBytes);
          if (!up) x_stage = s;
          const uint64_t db = umma_desc_sw128(smem_u32(ring + x_stage * kStageBytes) + kGABytes);
          if (dh) {
            const uint64_t da = umma_desc_mn_sw128(sa, kGBoxBytes);
#pragma unroll
            for (int k = 0; k < kGK / 16; ++k)
              f.umma(tm + (n & 1u) * kDuSlot, da + (uint64_t)(k * 128), db + (uint64_t)(k * 2), idesc | 1u << 15, (step | k) != 0 ? 1u : 0u);
            f.commit(&ctl.empty[s]);
          } else {
            const uint64_t da = umma_desc_sw128(sa);
            const uint32_t d = tm + (up ? 3 : 2) * kDuSlot;
#pragma unroll
            for (int k = 0; k < kGK / 16; ++k)
              f.umma(d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, (((step - k_blocks) >> 1) | k) != 0 ? 1u : 0u);
            if (up) {                          // both products with this block of x are behind: both stages are free
              f.commit(&ctl.empty[x_stage]);
              f.commit(&ctl.empty[s]);
            }
          }
          if (++s == kStages) { s = 0; ph ^= 1u; }
        }
        if (ok) f.commit(&ctl.acc_full[0]);
      }
      f.finish_products();
    }
  } else if (kSplit && warp >= 4) {
    PartSums<3> sums(ctl, staging, p.parts);
    const int thread = (warp - 4) * 32 + lane;
    uint32_t n = 0;
    for (int tile = f.first_tile; tile < total_tiles; tile += f.tile_step, ++n) {
      const RowTile t = walk.at(tile);
      const int sub = t.block / sub_blocks, unit0 = (t.block - sub * sub_blocks) * kTileM;
      if (!mbar_spin_progress_warp(&ctl.acc_full[0], n & 1u, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk)) break;
      tc_fence_after_sync();
      const uint32_t slots[3] = {(n & 1u) * kDuSlot, 2 * kDuSlot, 3 * kDuSlot};
      if (!sums.write(n, t.n, slots, abort_flag, p.dev_status)) break;
      if (lane == 0) {
        mbar_arrive(&ctl.acc_empty[n & 1u]);
        mbar_arrive(&ctl.u_empty);
      }
      if (!sums.publish(n, abort_flag, p.dev_status)) break;
      const int items = t.valid * (kGM / 4), to = items * (sums.part + 1) / p.parts;
      for (int i = items * sums.part / p.parts + thread; i < to; i += 256) {
        const int row = i / (kGM / 4), u = i % (kGM / 4) * 4, unit = unit0 + u;
        if (unit >= p.I) continue;
        float4 s[3];
        sums.joined(row, u, s);
        float vh[4], v1[4], v3[4];
        expert_unit(s[1].x, s[2].x, s[0].x, &vh[0], &v1[0], &v3[0]);
        expert_unit(s[1].y, s[2].y, s[0].y, &vh[1], &v1[1], &v3[1]);
        expert_unit(s[1].z, s[2].z, s[0].z, &vh[2], &v1[2], &v3[2]);
        expert_unit(s[1].w, s[2].w, s[0].w, &vh[3], &v1[3], &v3[3]);
        const size_t I = (size_t)p.I, ld = I * p.subs, at = (size_t)(t.row0 + row) * ld + I * sub + unit;
        uint16_t* du = p.du + (size_t)(t.row0 + row) * 2 * ld + 2 * I * sub + unit;
        *reinterpret_cast<uint2*>(p.h + at) = make_uint2(pack_bf16x2(vh[0], vh[1]), pack_bf16x2(vh[2], vh[3]));
        *reinterpret_cast<uint2*>(du) = make_uint2(pack_bf16x2(v1[0], v1[1]), pack_bf16x2(v1[2], v1[3]));
        *reinterpret_cast<uint2*>(du + I) = make_uint2(pack_bf16x2(v3[0], v3[1]), pack_bf16x2(v3[2], v3[3]));
      }
      sums.release();
    }
  } else if (warp >= 4) {
    const int q = warp & 3;
    unsigned char* buf = staging + (warp - 4) * 3 * kPieceBytes;
    uint32_t n = 0;
    for (int tile = f.first_tile; tile < total_tiles; tile += f.tile_step, ++n) {
      const RowTile t = walk.at(tile);
      if (!mbar_spin_progress_warp(&ctl.acc_full[0], n & 1u, abort_flag, &ctl.progress, p.dev_status, kWaitLimitClk)) break;
      tc_fence_after_sync();
      const uint32_t lanes = ctl.tmem_base + ((uint32_t)(q * 32) << 16), t_dh = lanes + (n & 1u) * kDuSlot, t_u = lanes + 2 * kDuSlot;
      const int sub = t.block / sub_blocks, col0 = (t.block - sub * sub_blocks) * kTileM + (int)f.rank * kGM + q * 32;
      if (col0 < p.I)
#pragma unroll 1
        for (int r = ((warp - 4) >> 2) * 32; r < t.valid; r += 64) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t at = ((uint32_t)half << 20) + (uint32_t)r;            // 16 lanes further
            uint32_t d[16], u1[16], u3[16], wh[8], w1[8], w3[8];
            tmem_ld_16x256b_x4(t_dh + at, d);
            tmem_ld_16x256b_x4(t_u + at, u1);
            tmem_ld_16x256b_x4(t_u + kDuSlot + at, u3);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float vh[2], v1[2], v3[2];
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                expert_unit(__uint_as_float(u1[2 * i + k]), __uint_as_float(u3[2 * i + k]), __uint_as_float(d[2 * i + k]), &vh[k], &v1[k], &v3[k]);
              }
              wh[i] = pack_bf16x2(vh[0], vh[1]);
              w1[i] = pack_bf16x2(v1[0], v1[1]);
              w3[i] = pack_bf16x2(v3[0], v3[1]);
            }
            piece_store_half(buf, half, lane, wh);
            piece_store_half(buf + kPieceBytes, half, lane, w1);
            piece_store_half(buf + 2 * kPieceBytes, half, lane, w3);
          }
          __syncwarp();
          const size_t I = (size_t)p.I, ld = I * p.subs;
          uint16_t* du = p.du + 2 * I * sub;
          piece_copy_out(buf, p.h + I * sub, ld, t.row0 + r, t.valid - r, col0, p.I, lane);
          piece_copy_out(buf + kPieceBytes, du, 2 * ld, t.row0 + r, t.valid - r, col0, p.I, lane);
          piece_copy_out(buf + 2 * kPieceBytes, du + I, 2 * ld, t.row0 + r, t.valid - r, col0, p.I, lane);
          __syncwarp();
        }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        f.arrive_leader(&ctl.acc_empty[n & 1u]);
        f.arrive_leader(&ctl.u_empty);
      }
    }
  }
  if (kSplit) cluster_sync_all();        // no CTA leaves while another reads its sums
  f.close();
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

template <bool kPair, typename... KArgs, typename... Args>
moe_status launch_grouped(void (*kernel)(KArgs...), size_t smem, PerDeviceOnce& attr_set, cudaStream_t stream, Args... args) {
  if (!ensure_dynamic_smem(kernel, smem, attr_set)) return MOE_ERR_CUDA;
  const unsigned grid = (unsigned)(kPair ? sm_count() & ~1 : sm_count());
  return launch_dependent_cluster(kernel, dim3(grid), dim3(kGThreads), smem, stream, dim3(kPair ? 2 : 1, 1, 1), args...) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}
constexpr size_t kMostSmem = 232448;     // the 227 KB that a CTA may use

// Boxes of 16 .. 16 count rows: those that the kernel may pick from.
bool row_maps(RowMaps& m, const void* base, int cols, int rows, int count) {
  bool ok = true;
  for (int i = 0; i < count; ++i) ok = ok && make_tmap(&m.m[i], base, (uint64_t)cols, (uint64_t)rows, 0, (uint64_t)cols, 0, 16u * (i + 1));
  return ok;
}

// Pairs where the groups have more than 64 rows on average (a single CTA's tile takes 64).
bool pair_rows(int64_t rows, int groups) { return rows > 64ll * groups; }

template <bool kT, bool kPair>
moe_status launch_rows_variant(const RowsParams& p, const CUtensorMap& w, const RowMaps& m, cudaStream_t stream) {
  constexpr size_t smem = RowsRing<kPair>::kBytes + 8 * kPieceBytes + sizeof(GroupedCtl) + 1024;
  static_assert(smem <= kMostSmem, "ring, staging and control block exceed what a CTA may use");
  static PerDeviceOnce attr_set;
  return launch_grouped<kPair>(rows_kernel<kT, kPair, false>, smem, attr_set, stream, p, w, m);
}
// Clusters that are resident at once, with some to spare: 15 of eight and 33 of four were, 16 and 34 ran twice as long.
int cluster_fit(int parts) { return parts == 8 ? 14 : parts == 4 ? 32 : 72; }

template <bool kT>
moe_status launch_rows_split(const RowsParams& p, const CUtensorMap& w, const RowMaps& m, cudaStream_t stream) {
  constexpr size_t smem = (size_t)kRowsSplitStages * RowsRing<false>::kStageBytes + PartSums<1>::kBytes + sizeof(GroupedCtl) + 1024;
  static_assert(smem <= kMostSmem, "ring, sums and control block exceed what a CTA may use");
  static PerDeviceOnce attr_set;
  if (!ensure_dynamic_smem(rows_kernel<kT, false, true>, smem, attr_set)) return MOE_ERR_CUDA;
  return launch_dependent_cluster(rows_kernel<kT, false, true>, dim3((unsigned)(cluster_fit(p.parts) * p.parts)), dim3(kGThreads), smem, stream,
                                  dim3((unsigned)p.parts, 1, 1), p, w, m) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}
// CTAs that share a tile's contraction, 1: none do.  A block of 64 along it costs a CTA about as long as 24 KB of loads, whatever its rows; a round
// of tiles that are joined costs 3 us more.  The estimate is of even segments, so a fifth has to be gained.
int rows_parts(int64_t P, int64_t E, int64_t k_len, int64_t n_cols, bool pair) {
  const int64_t k_blocks = (k_len + kGK - 1) / kGK, touched = P < E ? P : E, rows = (P + touched - 1) / touched;
  const auto rounds = [&](int64_t most, int64_t tile_m, int64_t resident) {
    return (touched * ((rows + most - 1) / most) * ((n_cols + tile_m - 1) / tile_m) + resident - 1) / resident;
  };
  // in tenths of a microsecond
  double best = 0.8 * k_blocks * (pair ? rounds(256, 2 * kGM, 74) * (1.3 + (rows < 256 ? rows : 256) / 128.0) : rounds(64, kGM, 148) * 1.3);
  int parts = 1;
  for (int k = 2; k <= kSplitMost && k <= k_blocks; k *= 2) {
    const double c = rounds(kPartRows, kGM, cluster_fit(k)) * ((k_blocks + k - 1) / k * 1.3 + 30);
    if (c < best) { best = c; parts = k; }
  }
  return parts;
}

// out [P, n] = rows [P, k] times W_e^T, W [E, n, k] (kT: times W_e, W [E, k, n])
template <bool kT>
moe_status launch_rows(int P, int k, int n, int E, const uint16_t* rows, const int32_t* offsets, const uint16_t* W, uint16_t* out,
                       int32_t* dev_status, cudaStream_t stream, GroupedStart start = GroupedStart::kAfterLast) {
  RowMaps m{};
  CUtensorMap w;
  const bool pair = pair_rows(P, E);
  bool ok = row_maps(m, rows, k, P, (pair ? RowsRing<true>::kMost / 2 : RowsRing<false>::kMost) / 16);
  if (kT) ok = ok && make_tmap(&w, W, (uint64_t)n, (uint64_t)k, (uint64_t)E, (uint64_t)n, (uint64_t)n * k, 64);
  else ok = ok && make_tmap(&w, W, (uint64_t)k, (uint64_t)n, (uint64_t)E, (uint64_t)k, (uint64_t)n * k, kGM);
  if (!ok) return MOE_ERR_CUDA;
  RowsParams p{offsets, E, P, n, k, out, dev_status, start, 1};
  p.parts = rows_parts(P, E, k, n, pair);
  if (p.parts > 1) return launch_rows_split<kT>(p, w, m, stream);
  return pair ? launch_rows_variant<kT, true>(p, w, m, stream) : launch_rows_variant<kT, false>(p, w, m, stream);
}

template <bool kPair, bool kF32>
moe_status launch_weights_variant(const WeightsParams& p, const WeightsMaps2& m, cudaStream_t stream) {
  constexpr size_t smem = WeightsRing<kPair, kF32>::kBytes + 8 * WeightsRing<kPair, kF32>::kStageOut + sizeof(GroupedCtl) + 1024;
  static_assert(smem <= kMostSmem, "ring, staging and control block exceed what a CTA may use");
  static PerDeviceOnce attr_set;
  return launch_grouped<kPair>(weights_kernel<kPair, kF32>, smem, attr_set, stream, p, m);
}

// out [E, m, n] = a^T b over the rows of each segment; a [P, m], b [P, n] with ldb elements from row to row
struct WeightsOperands {
  const uint16_t* a;
  const uint16_t* b;
  int m, n;
  int64_t ldb;
  void* out;
};
// How a product's tiles and rows are cut for split_weights_kernel; parts 1: they are not.  With few tiles a CTA's loads bound both kernels, about
// 0.13 us for a box of 8 KB (a little less in a pair, which loads four boxes a block), however few SMs load; the hand-over costs 2.5 us,
// 20 boxes.  Against measurements, above and split (us): one group of 512 rows, 512 x 512, 7.6 and 7.7; two of 750, 256 x 256, 11.4 and 9.1; one of
// 2048, 1024 x 1024, 14.6 and 12.6; one of 16 384, 64 x 64, 76.6 and 13.6.
struct SplitPlan { int parts, tile_n; };
SplitPlan split_plan(int64_t P, int E, int64_t m, int64_t n) {
  const int64_t blocks = ((E > 1 ? 2 : 1) * P / E + kGK - 1) / kGK, m_blocks = (m + kGM - 1) / kGM;       // of a long segment: twice the average
  const auto boxes_of = [&](int64_t tile_n) { return (m > 64 ? 2 : 1) + ((n < tile_n ? n : tile_n) + 63) / 64; };
  const bool pair = m > kGM;
  const int64_t whole_tiles = E * (pair ? (m_blocks + 1) / 2 : m_blocks) * ((n + kGN - 1) / kGN), resident = pair ? 74 : 148;
  double best = (double)((whole_tiles + resident - 1) / resident) * blocks * (pair ? 3.4 : (double)boxes_of(kGN));
  SplitPlan plan{1, kGN};
  for (int tile_n = 64; tile_n <= kGN; tile_n *= 2)
    for (int parts = 2; parts <= kSplitMost; parts *= 2) {
      const int64_t tiles = E * m_blocks * ((n + tile_n - 1) / tile_n), fit = cluster_fit(parts);
      const double cost = (double)((blocks + parts - 1) / parts * boxes_of(tile_n) + 20);
      if (tiles > fit || cost >= best) continue;
      best = cost;
      plan = {parts, tile_n};
    }
  return plan;
}
moe_status launch_split_weights(int P, int E, const int32_t* offsets, const WeightsOperands& q, const SplitPlan& plan, bool f32, bool add,
                                int32_t* dev_status, cudaStream_t stream) {
  SplitMaps m;
  bool ok = true;
  for (int i = 0; i < kGHeights; ++i)
    ok = ok && make_tmap(&m.a[i], q.a, (uint64_t)q.m, (uint64_t)P, 0, (uint64_t)q.m, 0, 1u << i) &&
         make_tmap(&m.b[i], q.b, (uint64_t)q.n, (uint64_t)P, 0, (uint64_t)q.ldb, 0, 1u << i);
  if (!ok) return MOE_ERR_CUDA;
  const int m_blocks = (q.m + kGM - 1) / kGM, n_blocks = (q.n + plan.tile_n - 1) / plan.tile_n, parts = plan.parts;
  const SplitParams p{offsets, E, P, q.m, q.n, parts, m_blocks, n_blocks, plan.tile_n, add, q.out, dev_status};
  constexpr size_t smem = kSplitRing + sizeof(GroupedCtl) + 1024;
  static_assert(smem <= kMostSmem, "ring and control block exceed what a CTA may use");
  static PerDeviceOnce once[2];
  auto kernel = f32 ? split_weights_kernel<true> : split_weights_kernel<false>;
  if (!ensure_dynamic_smem(kernel, smem, once[f32])) return MOE_ERR_CUDA;
  return launch_dependent_cluster(kernel, dim3((unsigned)(E * m_blocks * n_blocks * parts)), dim3(kGThreads), smem, stream,
                                  dim3((unsigned)parts, 1, 1), p, m) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}
moe_status launch_weights(int P, int E, const int32_t* offsets, const WeightsOperands* q, int problems, bool f32, bool add, int32_t* dev_status,
                          cudaStream_t stream, GroupedStart start = GroupedStart::kAfterLast) {
  WeightsMaps2 m;
  WeightsParams p{offsets, E, P, problems, {}, add, dev_status, start};
  bool ok = true, pair = false;
  for (int k = 0; k < problems; ++k) {
    WeightsMaps& w = m.q[k];
    for (int i = 0; i < kGHeights; ++i)
      ok = ok && make_tmap(&w.a[i], q[k].a, (uint64_t)q[k].m, (uint64_t)P, 0, (uint64_t)q[k].m, 0, 1u << i) &&
           make_tmap(&w.b[i], q[k].b, (uint64_t)q[k].n, (uint64_t)P, 0, (uint64_t)q[k].ldb, 0, 1u << i);
    if (f32) ok = ok && make_tmap_f32(&w.out, q[k].out, (uint64_t)q[k].n, (uint64_t)q[k].m, (uint64_t)E, 32);
    else w.out = w.a[0];
    p.q[k] = {q[k].m, q[k].n, q[k].out};
    pair = pair || q[k].m > kGM;
  }
  if (!ok) return MOE_ERR_CUDA;
  if (problems == 1) m.q[1] = m.q[0];
  if (pair) return f32 ? launch_weights_variant<true, true>(p, m, stream) : launch_weights_variant<true, false>(p, m, stream);
  return f32 ? launch_weights_variant<false, true>(p, m, stream) : launch_weights_variant<false, false>(p, m, stream);
}

template <bool kPair>
moe_status launch_du(const DuParams& p, const CUtensorMap& w13, const CUtensorMap& w2, const RowMaps& x, const RowMaps& dy, cudaStream_t stream) {
  constexpr size_t smem = DuRing<kPair>::kBytes + 8 * 3 * kPieceBytes + sizeof(GroupedCtl) + 1024;
  static_assert(smem <= kMostSmem, "ring, staging and control block exceed what a CTA may use");
  static PerDeviceOnce attr_set;
  return launch_grouped<kPair>(expert_du_kernel<kPair, false>, smem, attr_set, stream, p, w13, w2, x, dy);
}

// CTAs that share a tile's contraction, 1: none do.
int du_parts(int64_t P, const DuParams& p, bool pair) {
  const int64_t k_blocks = p.H / kGK, touched = P < p.E ? P : p.E, rows = (P + touched - 1) / touched;
  // What bounds a CTA is what it loads, in KB; a round of tiles that are joined costs as much as 150 more (2 us).  The estimate is of even segments,
  // so a fifth has to be gained.
  const auto cost = [&](int64_t most, int64_t tile_m, int64_t resident, int64_t parts, int64_t more) {
    const int64_t tiles = touched * ((rows + most - 1) / most) * ((p.I + tile_m - 1) / tile_m) * p.subs, n = rows < most ? rows : most;
    return (tiles + resident - 1) / resident * ((k_blocks + parts - 1) / parts * (48 + n * (tile_m == kGM ? 256 : 128) / 1024) + more);
  };
  int64_t best = (pair ? cost(128, 2 * kGM, 74, 1, 0) : cost(64, kGM, 148, 1, 0)) * 4 / 5;
  int parts = 1;
  for (int k = 2; k <= kSplitMost && k <= k_blocks; k *= 2) {
    const int64_t c = cost(64, kGM, cluster_fit(k), k, 150);
    if (c < best) { best = c; parts = k; }
  }
  return parts;
}
moe_status launch_split_du(const DuParams& p, const CUtensorMap& w13, const CUtensorMap& w2, const RowMaps& x, const RowMaps& dy, cudaStream_t stream) {
  constexpr size_t smem = (size_t)kDuSplitStages * DuRing<false>::kStageBytes + PartSums<3>::kBytes + sizeof(GroupedCtl) + 1024;
  static_assert(smem <= kMostSmem, "ring, sums and control block exceed what a CTA may use");
  static PerDeviceOnce attr_set;
  if (!ensure_dynamic_smem(expert_du_kernel<false, true>, smem, attr_set)) return MOE_ERR_CUDA;
  return launch_dependent_cluster(expert_du_kernel<false, true>, dim3((unsigned)(cluster_fit(p.parts) * p.parts)), dim3(kGThreads), smem, stream,
                                  dim3((unsigned)p.parts, 1, 1), p, w13, w2, x, dy) == cudaSuccess
             ? MOE_OK
             : MOE_ERR_CUDA;
}

}  // namespace

moe_status launch_grouped_gemm(const moe_grouped_shape* s, const uint16_t* x, const int32_t* offsets, const uint16_t* W, uint16_t* y,
                               int32_t* dev_status, cudaStream_t stream) {
  return launch_rows<false>(s->P, s->K, s->M, s->E, x, offsets, W, y, dev_status, stream);
}
moe_status launch_grouped_gemm_dx(const moe_grouped_shape* s, const uint16_t* dy, const int32_t* offsets, const uint16_t* W, uint16_t* dx,
                                  int32_t* dev_status, cudaStream_t stream) {
  return launch_rows<true>(s->P, s->M, s->K, s->E, dy, offsets, W, dx, dev_status, stream);
}
moe_status launch_grouped_gemm_dw(const moe_grouped_shape* s, const uint16_t* dy, const uint16_t* x, const int32_t* offsets, void* dW,
                                  int32_t* dev_status, cudaStream_t stream) {
  const WeightsOperands q{dy, x, s->M, s->K, s->K, dW};
  const bool f32 = (s->flags & MOE_GROUPED_DW_FP32) != 0, add = (s->flags & MOE_GROUPED_DW_ADD) != 0;
  const SplitPlan plan = split_plan(s->P, s->E, s->M, s->K);
  if (plan.parts > 1) return launch_split_weights(s->P, s->E, offsets, q, plan, f32, add, dev_status, stream);
  return launch_weights(s->P, s->E, offsets, &q, 1, f32, add, dev_status, stream);
}

moe_status launch_ffn_backward(const FfnBackwardArgs& a) {
  const size_t w = (size_t)a.E * a.S * a.H * a.I * 2;
  if (a.rows == 0) {        // no pairs: the weights' gradients are zero
    if (a.dW13 != nullptr && cudaMemsetAsync(a.dW13, 0, 2 * w, a.stream) != cudaSuccess) return MOE_ERR_CUDA;
    if (a.dW2 != nullptr && cudaMemsetAsync(a.dW2, 0, w, a.stream) != cudaSuccess) return MOE_ERR_CUDA;
    return MOE_OK;
  }
  const int P = (int)a.rows, H = a.H, I = a.I, E = a.E, S = a.S;
  GroupedStart start = GroupedStart::kAfterLast;
  const uint16_t* x_list = a.x;
  if (a.perm_token != nullptr) {
    const int most = sm_count() * 8, blocks = (P + 7) / 8;
    if (launch_dependent(list_rows_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, a.stream, 1, reinterpret_cast<const uint4*>(a.x),
                         a.perm_token, a.T, H / 8, P, reinterpret_cast<uint4*>(a.x_rows), a.dev_status) != cudaSuccess)
      return MOE_ERR_CUDA;
    start = GroupedStart::kBesideLast;
    x_list = a.x_rows;
  }
  static_assert(DuRing<true>::kMost / 2 == 64 && DuRing<false>::kMost == 64, "boxes of 16 to 64 rows");
  RowMaps mx{}, mdy{};
  CUtensorMap w13, w2;
  bool ok = row_maps(mx, x_list, H, P, 4) && row_maps(mdy, a.d_y, H, P, 4);        // a CTA loads 64 rows at most, in a pair too
  // W1 and W3 of a (sub-)expert as two matrices of I rows each
  ok = ok && make_tmap(&w13, a.W13, (uint64_t)H, (uint64_t)I, 2ull * E * S, (uint64_t)H, (uint64_t)I * H, kGM);
  ok = ok && make_tmap(&w2, a.W2, (uint64_t)I, (uint64_t)H, (uint64_t)E * S, (uint64_t)I, (uint64_t)H * I, 64);
  if (!ok) return MOE_ERR_CUDA;
  DuParams p{a.offsets, E, P, H, I, S, a.h, a.du, a.dev_status, start, 1};
  p.parts = du_parts(P, p, pair_rows(P, E));
  moe_status r = p.parts > 1       ? launch_split_du(p, w13, w2, mx, mdy, a.stream)
                 : pair_rows(P, E) ? launch_du<true>(p, w13, w2, mx, mdy, a.stream)
                                   : launch_du<false>(p, w13, w2, mx, mdy, a.stream);
  // all below need h and du alone: the first waits, the others start beside it
  start = GroupedStart::kAfterLast;
  if (r == MOE_OK && a.dx != nullptr) {
    r = launch_rows<true>(P, 2 * S * I, H, E, a.du, a.offsets, a.W13, a.dx, a.dev_status, a.stream);
    start = GroupedStart::kBesideLast;
  }
  // dW13 of a group is one matrix of S*2I rows, dW2 one for each sub-expert; two a launch
  WeightsOperands q[2];
  int n = 0;
  const int subs = a.dW2 != nullptr ? S : 0, total = subs + (a.dW13 != nullptr ? 1 : 0);
  for (int k = 0; r == MOE_OK && k < total; ++k) {
    const int sub = k - (total - subs);
    if (sub < 0) q[n++] = {a.du, x_list, 2 * S * I, H, H, a.dW13};
    else q[n++] = {a.d_y, a.h + (size_t)sub * I, H, I, (int64_t)S * I, a.dW2 + (size_t)sub * H * I};
    if (n < 2 && k + 1 < total) continue;
    r = launch_weights(P, E, a.offsets, q, n, false, false, a.dev_status, a.stream, start);
    start = GroupedStart::kBesideLast;
    n = 0;
  }
  return r;
}
