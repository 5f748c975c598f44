// Host-side builder of TMA tensor maps (cuTensorMapEncodeTiled through the runtime's driver entry point),
// shared by the expert GEMMs and the gate.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

// bf16 tensor [d2][d1][d0] (d0 contiguous; d2 == 0: two-dimensional), box {64, box1, 1}, 128-byte swizzle,
// out-of-range elements read as zero.  Strides in elements.  False when the driver refuses the map.
bool make_tmap(CUtensorMap* tm, const void* base, uint64_t d0, uint64_t d1, uint64_t d2, uint64_t stride1_elems,
               uint64_t stride2_elems, uint32_t box1);

// bf16 matrices [subs][halves][rows][K] (strides in elements, K contiguous) as a five-dimensional map with box
// {64, box_rows, halves, box_blocks, 1}: one load brings box_blocks consecutive 64-wide blocks of K, each stored as its own
// tile of halves x box_rows swizzled rows.  box_blocks > 1 needs K % 64 == 0 and takes the coordinates
// (0, row, 0, block, sub); box_blocks == 1 takes (column, row, 0, 0, sub).  Strides must be multiples of 8 elements.
struct KBlockedTensor {
  uint64_t K = 0, rows = 0, row_stride = 0;
  uint64_t halves = 1, half_stride = 8;
  uint64_t subs = 1, sub_stride = 8;
};
bool make_tmap_blocks(CUtensorMap* tm, const void* base, const KBlockedTensor& t, uint32_t box_rows, uint32_t box_blocks);
