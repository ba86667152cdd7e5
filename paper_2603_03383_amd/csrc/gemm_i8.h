// What the kernels of the 8-bit product (gemm_i8.hip, gemm_i8_tile.hip) share.
#pragma once
#include "i8.h"

namespace mdz {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
__device__ inline i32x4 mfma_i8(i32x4 a, i32x4 b, i32x4 c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }

// y[m][n] = sx[m] * sw[n] * sum_k X[m][k] * W[n][k]
struct I8Product {
  const int8_t* X;  // rows ldx bytes apart
  const float* sx;
  const uint8_t* W;  // packed codes (i8.h)
  const float* sw;
  void* Y;
  int M, N, K;
  int64_t ldx, kp;  // kp: padded features of a row of W
  int n_tiles;      // of W
};

// Writes four consecutive columns of a row.  The MFMAs are issued as W x X^T, so a lane holds such a quad; it leaves as one store wherever the row
// starts.  (An aligned quad beside a store per element is merged with it by the compiler, to three columns and one in fp32, two and two
// singles in binary16.  us so / unaligned: 1196 x 19319 x 310 binary16 54.4 / 36.8, 781 x 14784 x 1792 fp32 48.0 / 40.2, 200 x 6144 x 4096
// fp32 15.1 / 14.4; 1024 x 22016 x 4096 bf16, whose quads were whole, 101.6 / 102.3.)
template <typename TO>
__device__ inline void store_scaled(const I8Product& p, int row, int col, i32x4 sum, float sx) {
  struct Four {
    TO v[4];
  };
  typedef uint32_t Bits __attribute__((ext_vector_type(sizeof(Four) / 4)));
  typedef Bits Any __attribute__((aligned(1)));
  const float4 sw = *reinterpret_cast<const float4*>(p.sw + col);  // (padded to whole tiles)
  const Four f{{from_float<TO>((float)sum.x * (sx * sw.x)), from_float<TO>((float)sum.y * (sx * sw.y)),
                from_float<TO>((float)sum.z * (sx * sw.z)), from_float<TO>((float)sum.w * (sx * sw.w))}};
  TO* y = reinterpret_cast<TO*>(p.Y) + (int64_t)row * p.N + col;
  if (col + 4 <= p.N) {
    *reinterpret_cast<Any*>(y) = __builtin_bit_cast(Bits, f);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < p.N) y[e] = f.v[e];
  }
}

// ---- tiles of gemm_i8_tile.hip ---------------------------------------------------------------------
// `us_stage`: of one workgroup, us per 128 features; `us_all`: us per 128 features and workgroup where all CUs are busy, which is what
// the chip's fabric and caches deliver shared among them (from 11 TB/s for 256 x 192 tiles to 19 for 32 x 32, whose neighbours share more through the L2); `two`: two workgroups fit a CU's LDS.  See plan_i8.
struct I8Tile {
  int rows, cols, threads;
  bool two;
  float us_stage, us_all;
};
constexpr int kNumI8Tiles = 9;
extern const I8Tile kI8Tiles[kNumI8Tiles];
// workgroups of one part of the features, as a launch has them: in eights, one for each XCD
inline int64_t i8_tile_workgroups(const I8Tile& t, int M, int n_tiles) {
  const int64_t blocks = (int64_t)((M + t.rows - 1) / t.rows) * ((n_tiles * 16 + t.cols - 1) / t.cols);
  return (blocks + 7) / 8 * 8;
}
// The features in `splits` parts: more than one write their 32-bit sums to `partial` (splits x M x 16 n_tiles), and a second launch adds them.
int launch_i8_tile(int out_dtype, const I8Product& p, int tile, int splits, void* partial, hipStream_t st);
int launch_i8_tile_parts(const I8Product& p, int tile, int splits, void* partial, hipStream_t st);  // the first launch alone

}  // namespace mdz
