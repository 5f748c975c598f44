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

// fp32 tensor [d2][d1][d0], contiguous, box {32, box1, 1}: rows of 128 bytes with the 128-byte swizzle (stores).
bool make_tmap_f32(CUtensorMap* tm, const void* base, uint64_t d0, uint64_t d1, uint64_t d2, uint32_t box1);

// A five-dimensional bf16 tensor, innermost dimension first and contiguous; strides of dimensions 1 .. 4 in elements,
// multiples of 8.  Dimensions of size 1 take any such stride.
struct Tensor5 {
  uint64_t dim[5] = {1, 1, 1, 1, 1};
  uint64_t stride[4] = {8, 8, 8, 8};
};
// Its map: rows of row_bytes (128 or 64, box[0] elements) in shared memory with the swizzle of that width; elements out
// of range read as zero and are not written.  More dimensions than a matrix has let one load bring several tiles, each
// stored as its own run of rows: a weight's W1 and W3 rows, or consecutive 64-wide blocks of K (dim[0] = 64, K / 64 a
// dimension of stride 64, where 64 divides K).
bool make_tmap5(CUtensorMap* tm, const void* base, const Tensor5& t, const uint32_t (&box)[5], int row_bytes);
