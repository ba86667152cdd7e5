// Rows in 8-bit integers (include/medusa.h, "8-bit integer products"): the quantiser that every kernel writing such rows shares, and
// the packed layout of 8-bit weights.
#pragma once
#include "kernels.h"

namespace mdz {

// A launch counts its threads in 32 bits.
inline bool i8_launchable(int64_t workgroups, int threads) { return workgroups * threads <= (int64_t)UINT32_MAX; }

// ---- rows ------------------------------------------------------------------------------------------
// A row t in 8 bits: scale = max|t| / 127 (1 where that is zero), code = the integer nearest to t / scale, ties to even, clamped to
// +-127; decided in fp32.  A row that holds a NaN or an infinity has no scale: it becomes NaN and the codes 0, so that everything
// computed from the row is NaN, as it would be from the row itself.
constexpr float kI8Max = 127.f;
// max|t| is kept as its bits: as integers, the magnitudes of fp32 numbers order as the numbers do, then infinity, then NaN
__device__ inline uint32_t abs_bits(float t) { return __float_as_uint(t) & 0x7FFFFFFFu; }
struct I8Quantiser {
  float scale, inverse;
  bool bad, empty, plain;  // plain: the quotient below is good; else the division is left to the compiler's sequence for it
  __device__ explicit I8Quantiser(uint32_t amax_bits) {
    bad = amax_bits >= 0x7F800000u;
    const float s = __uint_as_float(amax_bits) / kI8Max;
    empty = s == 0.f;
    scale = bad ? __uint_as_float(0x7FC00000u) : empty ? 1.f : s;
    inverse = 1.f / scale;
    plain = scale >= 0x1p-100f && scale <= 0x1p100f;
  }
  // the scale of the row times `factor`: a row of zeros stands for zeros and keeps the scale 1, also where the factor is infinite
  __device__ inline float scale_times(float factor) const { return empty ? 1.f : scale * factor; }
  __device__ inline float code(float quotient) const { return __builtin_amdgcn_fmed3f(rintf(quotient), -kI8Max, kI8Max); }
  // The codes of W values, as numbers.  Three operations make the rounded quotient: a product with the rounded reciprocal, the rest it
  // leaves, which is exact, and the rest's share (1024 rows of 12800 with SwiGLU: 21.8 us with the
  // compiler's divisions, 20.2 so; 4000 plain rows of 1387: 10.1 / 8.9).
  template <int W>
  __device__ inline void round(const float (&t)[W], float (&c)[W]) const {
    if (plain) {
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const float q = t[e] * inverse;
        c[e] = code(fmaf(fmaf(-q, scale, t[e]), inverse, q));
      }
    } else {
#pragma unroll
      for (int e = 0; e < W; ++e) c[e] = bad ? 0.f : code(t[e] / scale);
    }
  }
};

// ---- packed weights --------------------------------------------------------------------------------
// Rows (output features) in tiles of 16, input features in k-steps of 64.  Memory order [tile][k-step][lane][16 codes]: one k-step of a
// tile is 1 KiB, the B operand of v_mfma_i32_16x16x64_i8 (lane l: row l % 16, features 64 ks + 16 (l / 16) .. +15), so a wave loads it
// with one instruction, and a tile is one contiguous stream.  Features are padded to 128 and rows to 16 with zeros.  One fp32 scale per
// (padded) row follows the codes of the whole matrix.
constexpr int kI8TileRows = MDZ_I8_TILE_ROWS;
constexpr int kI8KStep = 64;
constexpr int kI8MaxK = 131071;  // 128 * 128 * k < 2^31: no sum of products of codes leaves 32 bits
__host__ __device__ inline int64_t i8_padded_k(int64_t k) { return (k + 127) / 128 * 128; }
__host__ __device__ inline int64_t i8_padded_rows(int64_t n) { return (n + kI8TileRows - 1) / kI8TileRows * kI8TileRows; }
__host__ __device__ inline int64_t i8_scales_offset(int64_t n, int64_t k) { return i8_padded_rows(n) * i8_padded_k(k); }  // bytes
__host__ __device__ inline int64_t i8_packed_bytes(int64_t n, int64_t k) { return i8_scales_offset(n, k) + 4 * i8_padded_rows(n); }
// byte of (row n, feature k); kp = i8_padded_k
__host__ __device__ inline int64_t i8_index(int64_t n, int64_t k, int64_t kp) {
  return (n >> 4) * 16 * kp + (k >> 6) * 1024 + ((n & 15) + 16 * ((k >> 4) & 3)) * 16 + (k & 15);
}

// ---- a layer's products and norms (medusa_api.hip) ---------------------------------------------------
// A product whose features were cut into parts, as its consumer adds it up: y[m][n] = sx[m] * sw[n] * sum of parts[s][m][n], s < n.  n == 0: the
// product is finished.  (Of 149 products of 17 .. 700 rows with their norm, six or eight parts were the best for few: taking them too would make the best time 0.2 % less
// on average, 10 % at most; the norm then holds twice the registers.)
constexpr int kI8MaxParts = 4;
struct I8Sums {
  const int32_t* parts;
  int n, ld;
  int64_t stride;
  const float* sx;
  const float* sw;
};
// medusa_linear_i8 into y, or, where that is faster, parts in ws and no second launch, which stand for bit for bit the same numbers
int launch_linear_i8_parts(const int8_t* codes, const float* scales, const void* packed, int M, int N, int K, float* y, void* ws, int64_t ws_bytes,
                           I8Sums* sums, hipStream_t st);
int64_t linear_i8_parts_bytes(int M, int N, int K);
// medusa_residual_rmsnorm_i8 in place with such a product as the update (delta where sums.n == 0), the same x and codes bit for bit; parts need
// d <= kI8MaxPartsWidth and a multiple of four
constexpr int kI8MaxPartsWidth = 16384;
int launch_residual_rmsnorm_i8(int dtype, float* x, const float* delta, const I8Sums& sums, const void* gain, float eps, int rows, int d,
                               int8_t* codes, float* scales, hipStream_t st);

}  // namespace mdz
