// Product of rows in 8 bits with packed 8-bit weights: y[m][n] = sx[m] * sw[n] * sum_k cx[m][k] * cw[n][k], sums in 32-bit integers.
#include "i8.h"

namespace mdz {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// 16 codes of a row of K from feature k on (any alignment); features beyond K come as zeros
__device__ inline i32x4 load_codes(const int8_t* row, int k, int K) {
  typedef i32x4 i32x4_any __attribute__((aligned(1)));
  if (k + 16 <= K) return *reinterpret_cast<const i32x4_any*>(row + k);
  i32x4 v{0, 0, 0, 0};
  for (int j = 0; j < K - k; ++j) v[j >> 2] |= (int32_t)(uint8_t)row[k + j] << (8 * (j & 3));
  return v;
}

// A workgroup of four waves makes MT 16-row tiles x one 16-column tile: the waves share the k-steps and add their sums through LDS.
template <int MT, typename TO>
__global__ void __launch_bounds__(256) gemm_i8_kernel(const int8_t* __restrict__ X, const float* __restrict__ sx,
                                                      const uint8_t* __restrict__ Wp, const float* __restrict__ sw, TO* __restrict__ Y,
                                                      int M, int N, int K, int64_t kp) {
  __shared__ i32x4 red[4][MT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row0 = blockIdx.y * MT * 16;
  const int n_steps = (K + kI8KStep - 1) / kI8KStep;
  const int8_t* xr[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) xr[i] = X + (int64_t)min(row0 + i * 16 + (lane & 15), M - 1) * K;
  const uint8_t* w = Wp + (int64_t)blockIdx.x * 16 * kp + lane * 16;
  i32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = i32x4{0, 0, 0, 0};
  for (int ks = wave; ks < n_steps; ks += 4) {
    const i32x4 b = *reinterpret_cast<const i32x4*>(w + (int64_t)ks * 1024);
#pragma unroll
    for (int i = 0; i < MT; ++i)
      acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(load_codes(xr[i], ks * kI8KStep + 16 * (lane >> 4), K), b, acc[i], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) red[wave][i][lane] = acc[i];
  __syncthreads();
  for (int p = threadIdx.x; p < MT * 64; p += 256) {
    const int i = p >> 6, l = p & 63, col = blockIdx.x * 16 + (l & 15);
    const i32x4 s = red[0][i][l] + red[1][i][l] + red[2][i][l] + red[3][i][l];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = row0 + i * 16 + 4 * (l >> 4) + e;
      if (row < M && col < N) Y[(int64_t)row * N + col] = from_float<TO>((float)s[e] * (sx[row] * sw[col]));
    }
  }
}

template <typename TO>
static int launch_gemm_i8_t(const int8_t* X, const float* sx, const void* Wp, int M, int N, int K, TO* Y, hipStream_t st) {
  const int64_t kp = i8_padded_k(K);
  const float* sw = (const float*)((const char*)Wp + i8_scales_offset(N, K));
  const unsigned n_tiles = (unsigned)(i8_padded_rows(N) / kI8TileRows);
  auto run = [&](auto kernel, int rows) {
    launch_timed(PROF_GEMM_I8, kernel, dim3(n_tiles, (M + rows - 1) / rows), 256, 0, st, X, sx, (const uint8_t*)Wp, sw, Y, M, N, K, kp);
  };
  if (M <= 16) run(gemm_i8_kernel<1, TO>, 16);
  else if (M <= 32) run(gemm_i8_kernel<2, TO>, 32);
  else run(gemm_i8_kernel<4, TO>, 64);
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

}  // namespace mdz

using namespace mdz;

extern "C" {
#pragma GCC visibility push(default)

int64_t medusa_linear_i8_workspace_bytes(int M, int N, int K) {
  MDZ_REQUIRE(M >= 0 && N > 0 && K > 0, MDZ_EINVAL, "linear_i8: [%d,%d] x [%d,%d]", M, K, N, K);
  MDZ_REQUIRE(K <= kI8MaxK, MDZ_EUNSUPPORTED, "linear_i8: up to %d input features, whose 32-bit sums cannot overflow (%d)", kI8MaxK, K);
  return 0;
}

int medusa_linear_i8(const int8_t* codes, const float* scales, const void* packed, int M, int N, int K, int out_dtype, void* y, void* ws,
                     int64_t ws_bytes, void* stream) {
  MDZ_REQUIRE(dtype_ok(out_dtype), MDZ_EINVAL, "linear_i8: bad dtype %d", out_dtype);
  const int64_t need = medusa_linear_i8_workspace_bytes(M, N, K);
  if (need < 0) return (int)need;
  if (M == 0) return MDZ_OK;
  MDZ_REQUIRE(codes && scales && packed && y, MDZ_EINVAL, "linear_i8: NULL pointer");
  MDZ_REQUIRE((reinterpret_cast<uintptr_t>(packed) & 15) == 0, MDZ_EINVAL, "linear_i8: the packed matrix must start on 16 bytes");
  MDZ_REQUIRE(reinterpret_cast<uintptr_t>(scales) % 4 == 0 && reinterpret_cast<uintptr_t>(y) % elem_bytes(out_dtype) == 0, MDZ_EINVAL,
              "linear_i8: a buffer is not aligned to its elements");
  MDZ_REQUIRE(ws_bytes >= need && (ws || need == 0), MDZ_EWORKSPACE, "linear_i8: workspace %lld < %lld bytes", (long long)ws_bytes,
              (long long)need);
  MDZ_WITH_ELEM(out_dtype, return launch_gemm_i8_t<E>(codes, scales, packed, M, N, K, (E*)y, (hipStream_t)stream));
}

#pragma GCC visibility pop
}  // extern "C"
