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

// How a product is cut: rows / 16 and tiles (a gated product's are half gate, half up) of a wave, waves of a workgroup, and for few rows the pieces of four of them that
// are loaded (0: the kernel of more rows).
struct I4Plan {
  int mt, nt, waves, xr;
};
// Whether q - z is made before the products (gemm_i4.h), and what a product costs by: 0 .. 2 groups of 128, 64 and 32 without zero points, 3 .. 5 with them,
// 6 and 7 groups of 64 and 32 whose zero points are subtracted.
__host__ __device__ constexpr bool i4_subtracts(bool f16, int groups_of_block) { return f16 && groups_of_block > 1; }
constexpr int i4_kind(bool f16, int groups_of_block, bool zeros) {
  const int g = groups_of_block == 1 ? 0 : groups_of_block == 2 ? 1 : 2;
  return !zeros ? g : i4_subtracts(f16, groups_of_block) ? 5 + g : 3 + g;
}
// The cuts for more than 16 rows: for how many rows, rows and tiles (of each matrix, if gated; 0: not gated) of a workgroup, blocks of features of a turn, and a
// turn's us on a full chip by kind: with one workgroup on a CU, and with two (0: the kernel of few rows, one).  A us of 0: the kind's registers spill, and other cuts are
// faster wherever this one would do (256 columns with bf16 zero points in groups of 64 took 1.85 and 4.1 us, which 128 columns with 1.22 and 1.55 beat at every size).
struct I4Cut {
  I4Plan plan;
  int least_rows, most_rows, rows, tiles, gate_tiles, features;
  float us[8], us_two[8];
};
constexpr I4Cut kI4Cuts[] = {
    {{2, 1, 8, 8}, 17, 32, 32, 1, 0, 8, {1.48f, 1.52f, 1.69f, 1.6f, 1.64f, 1.9f, 1.58f, 1.72f}, {}},
    {{2, 2, 8, 8}, 17, 32, 32, 2, 1, 8, {2.0f, 2.1f, 2.33f, 2.25f, 2.35f, 2.77f, 2.28f, 2.56f}, {}},
    {{2, 6, 4, 8}, 17, 32, 32, 6, 3, 4, {2.05f, 2.35f, 3.2f, 2.35f, 3.4f, 4.15f, 3.2f, 3.9f}, {}},
    {{4, 1, 8, 16}, 33, 1 << 30, 64, 1, 0, 8, {2.55f, 2.6f, 4.0f, 2.7f, 2.95f, 4.05f, 2.62f, 2.75f}, {}},
    {{4, 2, 8, 16}, 33, 1 << 30, 64, 2, 1, 8, {3.05f, 0.f, 0.f, 3.3f, 0.f, 0.f, 3.17f, 0.f}, {}},
    {{4, 6, 4, 16}, 33, 1 << 30, 64, 6, 3, 4, {3.05f, 3.7f, 0.f, 3.7f, 0.f, 0.f, 4.0f, 0.f}, {}},
    {{4, 2, 4, 0}, 17, 1 << 30, 64, 8, 4, 1, {0.95f, 1.0f, 1.16f, 1.15f, 1.22f, 1.54f, 1.04f, 1.2f}, {1.2f, 1.25f, 1.53f, 1.36f, 1.55f, 2.0f, 1.46f, 1.67f}},
    {{4, 4, 4, 0}, 17, 1 << 30, 64, 16, 8, 1, {1.38f, 1.43f, 2.05f, 1.55f, 0.f, 2.43f, 1.69f, 2.07f}, {2.12f, 2.35f, 2.87f, 2.33f, 0.f, 3.42f, 2.65f, 3.1f}},
};
// Whether there is a kernel with this cut for this kind.  Up to 16 rows groups of 32 take two tiles at most, with eight waves where zero points cost registers.
constexpr bool i4_built(const I4Plan& plan, int kind, bool gated) {
  const bool of_32 = kind == 2 || kind == 5 || kind == 7;
  if (plan.mt == 1 && gated && !of_32 && plan.nt == 2 && plan.waves == 4 && plan.xr == 4) return false;  // (9 to 16 rows of a gated product: four tiles beyond one per CU)
  if (plan.mt == 1) return !(of_32 && plan.nt == 4) && !(kind == 5 && plan.nt == 2 && plan.waves == 4) && (gated || kind == 5 || !(plan.nt == 2 && plan.waves == 8));
  for (const I4Cut& c : kI4Cuts)
    if (c.plan.mt == plan.mt && c.plan.nt == plan.nt && c.plan.waves == plan.waves && c.plan.xr == plan.xr) return c.us[kind] > 0.f;
  return false;
}

template <typename E, int G>
int launch_i4(const I4Product& p, bool zeros, bool gated, const I4Plan& plan, hipStream_t st);

}  // namespace mdz
