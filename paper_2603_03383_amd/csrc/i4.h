// Matrices in 4 bits (include/medusa.h, "4-bit weights"): the packed layout, and what the kernels of their products share.
#pragma once
#include "kernels.h"

namespace mdz {

// Rows (output features) in tiles of 16, input features in blocks of 128, 4 / 2 / 1 groups of 32 / 64 / 128 features in a block.
//   codes:  [tile][block][lane][16 bytes]: 1 KiB, four A operands of v_mfma_f32_16x16x32: word s of lane l holds row l % 16, features
//           32 s + 8 (l / 16) .. +7 of the block, so a wave loads a block with one instruction and a tile is one contiguous stream.
//   scales: [tile][block][16 rows][groups of the block], 16-bit; the products leave a lane with rows 4 (l / 16) .. +3, whose scales lie together.
//   zeros:  (only in matrices that have zero points) the same order, a byte each.
// The eight codes of a word stand in fields of four bits, feature e of them in field e / 2 + 4 (e % 2), and the word is rotated left by three (bf16) or
// six (binary16): two features are then one mask away from a pair of 16-bit floating numbers with the code at the top of the mantissa (see dequantise).
// Features are padded to 128 with codes equal to their zero points and rows to 16 with scales of zero.
constexpr int kI4TileRows = MDZ_I4_TILE_ROWS;
constexpr int kI4Block = 128;
constexpr int kI4MaxK = 1 << 24;  // features of a row: byte offsets inside a tile stay in 32 bits
__host__ __device__ inline int64_t i4_blocks(int64_t k) { return (k + kI4Block - 1) / kI4Block; }
__host__ __device__ inline int64_t i4_tiles(int64_t n) { return (n + kI4TileRows - 1) / kI4TileRows; }
__host__ __device__ inline int64_t i4_scales_offset(int64_t n, int64_t k) { return i4_tiles(n) * i4_blocks(k) * 1024; }  // bytes
__host__ __device__ inline int64_t i4_zeros_offset(int64_t n, int64_t k, int group) {
  return i4_scales_offset(n, k) + i4_tiles(n) * i4_blocks(k) * (32 * (kI4Block / group));
}
__host__ __device__ inline int64_t i4_packed_bytes(int64_t n, int64_t k, int group, bool zeros) {
  return i4_zeros_offset(n, k, group) + (zeros ? i4_tiles(n) * i4_blocks(k) * (16 * (kI4Block / group)) : 0);
}
inline bool i4_group_ok(int group) { return group == 32 || group == 64 || group == 128; }
// place of a word's feature e among the fields of four bits before the rotation
__host__ __device__ inline int i4_field(int e) { return (e >> 1) + 4 * (e & 1); }
template <typename E>
constexpr int kI4Rotation = __is_same(E, f16_t) ? 6 : 3;

// One matrix of a product.
struct I4Matrix {
  const uint8_t* codes;
  const uint8_t* scales;
  const uint8_t* zeros;
};
inline I4Matrix i4_matrix(const void* packed, int64_t n, int64_t k, int group) {
  const uint8_t* p = (const uint8_t*)packed;
  return I4Matrix{p, p + i4_scales_offset(n, k), p + i4_zeros_offset(n, k, group)};
}

// y[m][n] = sum_k x[m][k] w[n][k], or, where there is a second matrix, SiLU of that times the second's product
struct I4Product {
  const void* X;
  I4Matrix w[2];
  void* Y;
  int M, N, K, out_dtype;
  int64_t ldx;  // bytes from row to row of X
  int n_tiles, n_blocks;
  int nb_m, nb_n;  // workgroups of rows and of columns
};

// How a product is cut: rows / 16 and tiles (a gated product's are half gate, half up) of a wave, waves of rows (0: the kernel of few rows), of columns and of
// features, and for few rows the pieces of four of them that are loaded.
struct I4Plan {
  int mt, nt, wm, wn, wk, xr;
};
template <typename E, int G>
int launch_i4(const I4Product& p, bool zeros, bool gated, const I4Plan& plan, hipStream_t st);

}  // namespace mdz
