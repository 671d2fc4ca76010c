// The 4-bit paged cache's layout, shared by what writes, reads and attends to it.
#ifndef FC_MX_H_
#define FC_MX_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fc {

// Sixteen neighbouring slots, K and V of D columns, are a tile of 17 D bytes (2176 for 128 columns, 17 lines of 128 bytes).  A page is
// page_size / 16 tiles and pages follow each other, so that slot s is row s % 16 of tile s / 16 whatever the page size.
//   K codes   [16 rows][D / 2]              row-major: a lane of the score product takes D / 4 neighbouring columns of one row
//   V codes   [4 quads][16][4 rows][D / 32] a lane of the output product takes D / 16 columns of the four rows of a quad, one load
//   K scales  [D / 32][16 rows]
//   V scales  [4 quads][D / 32][4 rows]     the four rows' scales of a lane, one dword
// Codes: two a byte, the lower nibble the even column.  Scales: E of 2^(E - 127) for 32 columns.
template <int D> struct MxTile {
  static constexpr int kBytes = 17 * D, kV = 8 * D, kScales = 16 * D, kVScales = 16 * D + D / 2;
  __host__ __device__ static constexpr int k_code(int row, int byte) { return row * (D / 2) + byte; }
  __host__ __device__ static constexpr int v_code(int row, int n) { return kV + row / 4 * (2 * D) + n * (D / 8) + row % 4 * (D / 32); }
  __host__ __device__ static constexpr int k_scale(int row, int block) { return kScales + block * 16 + row; }
  __host__ __device__ static constexpr int v_scale(int row, int block) { return kVScales + row / 4 * (D / 8) + block * 4 + row % 4; }
};

// E of a block whose largest magnitude has these bits: the power of two that puts it below 7, the highest value that is not nearer to 8 than to
// 6 (from 7 on the next power holds it better, below it none does).  [2, 252]: every value is then a normal fp32 number.
// A block with an infinity or NaN has 255, which stands for NaN in all of it.
__device__ __forceinline__ uint32_t mx_scale(uint32_t top_bits) {
  const int e = (int)((top_bits + (1u << 21)) >> 23) - 2;
  return top_bits >= 0x7F800000u ? 255u : (uint32_t)min(max(e, 2), 252);
}

}  // namespace fc
#endif
