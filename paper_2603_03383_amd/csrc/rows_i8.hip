// Rows in 8 bits with one scale each: the residual's addition and RMSNorm, SwiGLU, plain rows, and the packing of 8-bit weights.
#include "i8.h"

namespace mdz {

template <typename T>
__device__ inline T block_reduce_256(T v, T* smem4, T (*op)(T, T)) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o, 64));
  if ((threadIdx.x & 63) == 0) smem4[threadIdx.x >> 6] = v;
  __syncthreads();
  return op(op(smem4[0], smem4[1]), op(smem4[2], smem4[3]));
}
__device__ inline float add_f(float a, float b) { return a + b; }
__device__ inline uint32_t max_u(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Where a kernel's rows come from: element i of row r as fp32, read once for the statistics and once for the codes.
template <typename E>
struct PlainRows {
  const E* src;
  int d;
  __device__ inline float first(int64_t r, int i, float&) const { return to_float(src[r * d + i]); }
  __device__ inline float again(int64_t r, int i) const { return to_float(src[r * d + i]); }
  __device__ inline float factor(float) const { return 1.f; }
};
template <typename E>
struct SwigluRows {
  const E* gate_up;
  int d;
  __device__ inline float first(int64_t r, int i, float&) const { return again(r, i); }
  __device__ inline float again(int64_t r, int i) const {
    const float g = to_float(gate_up[r * 2 * d + i]), u = to_float(gate_up[r * 2 * d + d + i]);
    return g / (1.f + expf(-g)) * u;
  }
  __device__ inline float factor(float) const { return 1.f; }
};
// x' = x + delta; the codes are those of x' * gain, because the norm's factor is positive and cancels; it goes into the scale
template <typename E, typename D>
struct NormRows {
  const float* x;
  const D* delta;
  const E* gain;
  float* x_out;
  int d;
  float eps;
  __device__ inline float sum(int64_t r, int i) const { return delta ? x[r * d + i] + to_float(delta[r * d + i]) : x[r * d + i]; }
  __device__ inline float first(int64_t r, int i, float& squares) const {
    const float v = sum(r, i);
    if (x_out) x_out[r * d + i] = v;  // (x_out may be x: the second reading is of x_out)
    squares += v * v;
    return v * to_float(gain[i]);
  }
  __device__ inline float again(int64_t r, int i) const { return (x_out ? x_out[r * d + i] : sum(r, i)) * to_float(gain[i]); }
  __device__ inline float factor(float squares) const { return 1.f / sqrtf(squares / (float)d + eps); }
};

template <typename Rows, typename E>
__global__ void __launch_bounds__(256) rows_i8_kernel(Rows in, int d, int8_t* codes, float* scales, E* values) {
  __shared__ float red_f[4];
  __shared__ uint32_t red_u[4];
  const int64_t r = blockIdx.x;
  float squares = 0.f;
  uint32_t amax = 0;
  for (int i = threadIdx.x; i < d; i += 256) amax = max_u(amax, abs_bits(in.first(r, i, squares)));
  amax = block_reduce_256(amax, red_u, max_u);
  squares = block_reduce_256(squares, red_f, add_f);
  const I8Quantiser q(amax);
  const float scale = q.scale * in.factor(squares);
  if (threadIdx.x == 0) scales[r] = scale;
  for (int i = threadIdx.x; i < d; i += 256) {
    const float c = q.round(in.again(r, i));
    codes[r * d + i] = (int8_t)c;
    if (values) values[r * d + i] = from_float<E>(c * scale);
  }
}

template <typename E, typename Rows>
static int launch_rows_i8(const Rows& in, int rows, int d, int8_t* codes, float* scales, void* values, hipStream_t st) {
  if (rows == 0) return MDZ_OK;
  launch_timed(PROF_ROWS_I8, rows_i8_kernel<Rows, E>, rows, 256, 0, st, in, d, codes, scales, (E*)values);
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

// One workgroup per row of the padded matrix: codes and scale of a source row, zeros for a row of the padding.
template <typename E>
__global__ void __launch_bounds__(256) pack_weight_i8_kernel(const E* src, int64_t n_rows, int64_t k, uint8_t* dst, int64_t kp,
                                                             int64_t first_row, float* scales) {
  __shared__ uint32_t red[4];
  const int64_t n = blockIdx.x, row = first_row + n;
  uint32_t amax = 0;
  if (n < n_rows)
    for (int64_t i = threadIdx.x; i < k; i += 256) amax = max_u(amax, abs_bits(to_float(src[n * k + i])));
  amax = block_reduce_256(amax, red, max_u);
  const I8Quantiser q(amax);
  if (threadIdx.x == 0) scales[row] = n < n_rows ? q.scale : 0.f;
  for (int64_t i = threadIdx.x; i < kp; i += 256)
    dst[i8_index(row, i, kp)] = (uint8_t)(n < n_rows && i < k ? (int8_t)q.round(to_float(src[n * k + i])) : 0);
}

__global__ void __launch_bounds__(256) pack_codes_i8_kernel(const int8_t* codes, const float* src_scales, int64_t n_rows, int64_t k,
                                                            uint8_t* dst, int64_t kp, int64_t first_row, float* scales) {
  const int64_t n = blockIdx.x, row = first_row + n;
  if (threadIdx.x == 0) scales[row] = n < n_rows ? src_scales[n] : 0.f;
  for (int64_t i = threadIdx.x; i < kp; i += 256) dst[i8_index(row, i, kp)] = (uint8_t)(n < n_rows && i < k ? codes[n * k + i] : 0);
}

static int check_pack_i8(const void* src, int64_t n_rows, int64_t k, const void* dst, int64_t dst_rows, int64_t tile_offset) {
  MDZ_REQUIRE(src && dst, MDZ_EINVAL, "pack i8: NULL pointer");
  MDZ_REQUIRE(n_rows > 0 && k > 0 && dst_rows >= n_rows && tile_offset >= 0, MDZ_EINVAL, "pack i8: bad sizes");
  MDZ_REQUIRE(k <= kI8MaxK && dst_rows <= INT32_MAX - kI8TileRows, MDZ_EUNSUPPORTED,
              "pack i8: [%lld,%lld]: up to %d input features, whose 32-bit sums cannot overflow, and 2^31 rows", (long long)dst_rows,
              (long long)k, kI8MaxK);
  MDZ_REQUIRE((reinterpret_cast<uintptr_t>(dst) & 15) == 0, MDZ_EINVAL, "pack i8: the packed matrix must start on 16 bytes");
  const int64_t end = tile_offset * kI8TileRows + i8_padded_rows(n_rows), all = i8_padded_rows(dst_rows);
  MDZ_REQUIRE(tile_offset <= all / kI8TileRows && end <= all, MDZ_ESHAPE, "pack i8: %lld rows at tile %lld exceed dst_rows %lld",
              (long long)n_rows, (long long)tile_offset, (long long)dst_rows);
  MDZ_REQUIRE(n_rows % kI8TileRows == 0 || end == all, MDZ_ESHAPE,
              "pack i8: n_rows %lld is not a multiple of the tile height %d and this is not the last matrix", (long long)n_rows, kI8TileRows);
  return MDZ_OK;
}

static bool on(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// src_bytes: of an element of src
static int check_rows_i8(const char* what, int dtype, const void* src, int src_bytes, int rows, int d, const void* codes,
                         const void* scales, const void* values) {
  MDZ_REQUIRE(dtype_ok(dtype), MDZ_EINVAL, "%s: bad dtype %d", what, dtype);
  MDZ_REQUIRE(rows >= 0 && d > 0 && d < (1 << 30), MDZ_EINVAL, "%s: rows %d, width %d", what, rows, d);
  MDZ_REQUIRE(rows == 0 || (src && codes && scales), MDZ_EINVAL, "%s: NULL pointer", what);
  MDZ_REQUIRE(on(src, src_bytes) && on(scales, 4) && on(values, elem_bytes(dtype)), MDZ_EINVAL, "%s: a buffer is not aligned to its elements",
              what);
  return MDZ_OK;
}

}  // namespace mdz

using namespace mdz;

extern "C" {
#pragma GCC visibility push(default)

int64_t medusa_packed_i8_bytes(int64_t n_rows, int64_t k) {
  MDZ_REQUIRE(n_rows > 0 && k > 0, MDZ_EINVAL, "packed_i8_bytes: sizes must be positive");
  MDZ_REQUIRE(k <= kI8MaxK && n_rows <= INT32_MAX - kI8TileRows, MDZ_EUNSUPPORTED,
              "packed_i8_bytes: up to %d input features, whose 32-bit sums cannot overflow, and 2^31 rows", kI8MaxK);
  return i8_packed_bytes(n_rows, k);
}

int medusa_pack_weight_i8(int dtype, const void* src, int64_t n_rows, int64_t k, void* dst, int64_t dst_rows, int64_t tile_offset,
                          void* stream) {
  MDZ_REQUIRE(dtype_ok(dtype), MDZ_EINVAL, "pack i8: bad dtype %d", dtype);
  int rc = check_pack_i8(src, n_rows, k, dst, dst_rows, tile_offset);
  if (rc) return rc;
  hipStream_t st = (hipStream_t)stream;
  ProfScope prof_(PROF_MISC, st);
  float* scales = (float*)((char*)dst + i8_scales_offset(dst_rows, k));
  MDZ_WITH_ELEM(dtype, (pack_weight_i8_kernel<E><<<(unsigned)i8_padded_rows(n_rows), 256, 0, st>>>(
                           (const E*)src, n_rows, k, (uint8_t*)dst, i8_padded_k(k), tile_offset * kI8TileRows, scales)));
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

int medusa_pack_codes_i8(const int8_t* codes, const float* scales, int64_t n_rows, int64_t k, void* dst, int64_t dst_rows,
                         int64_t tile_offset, void* stream) {
  MDZ_REQUIRE(scales, MDZ_EINVAL, "pack i8: NULL pointer");
  int rc = check_pack_i8(codes, n_rows, k, dst, dst_rows, tile_offset);
  if (rc) return rc;
  hipStream_t st = (hipStream_t)stream;
  ProfScope prof_(PROF_MISC, st);
  pack_codes_i8_kernel<<<(unsigned)i8_padded_rows(n_rows), 256, 0, st>>>(
      codes, scales, n_rows, k, (uint8_t*)dst, i8_padded_k(k), tile_offset * kI8TileRows,
      (float*)((char*)dst + i8_scales_offset(dst_rows, k)));
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

int medusa_quantize_rows_i8(int dtype, const void* src, int rows, int d, int8_t* codes, float* scales, void* values_opt, void* stream) {
  int rc = check_rows_i8("quantize_rows_i8", dtype, src, elem_bytes(dtype), rows, d, codes, scales, values_opt);
  if (rc) return rc;
  MDZ_WITH_ELEM(dtype, return launch_rows_i8<E>(PlainRows<E>{(const E*)src, d}, rows, d, codes, scales, values_opt, (hipStream_t)stream));
}

int medusa_swiglu_i8(int dtype, const void* gate_up, int rows, int ffn, int8_t* codes, float* scales, void* values_opt, void* stream) {
  int rc = check_rows_i8("swiglu_i8", dtype, gate_up, elem_bytes(dtype), rows, ffn, codes, scales, values_opt);
  if (rc) return rc;
  MDZ_WITH_ELEM(dtype, return launch_rows_i8<E>(SwigluRows<E>{(const E*)gate_up, ffn}, rows, ffn, codes, scales, values_opt,
                                                (hipStream_t)stream));
}

int medusa_residual_rmsnorm_i8(int dtype, const float* x, const void* delta_opt, int delta_dtype, const void* gain, float eps, int rows,
                               int d, float* x_out_opt, int8_t* codes, float* scales, void* values_opt, void* stream) {
  int rc = check_rows_i8("residual_rmsnorm_i8", dtype, x, 4, rows, d, codes, scales, values_opt);
  if (rc) return rc;
  MDZ_REQUIRE(rows == 0 || gain, MDZ_EINVAL, "residual_rmsnorm_i8: NULL pointer");
  MDZ_REQUIRE(!delta_opt || delta_dtype == MDZ_FP32 || delta_dtype == dtype, MDZ_EINVAL,
              "residual_rmsnorm_i8: delta is fp32 or of the gains' type (delta_dtype %d, dtype %d)", delta_dtype, dtype);
  MDZ_REQUIRE(eps >= 0.f, MDZ_EINVAL, "residual_rmsnorm_i8: eps must not be negative");
  MDZ_REQUIRE(on(gain, elem_bytes(dtype)) && on(x_out_opt, 4) && (!delta_opt || on(delta_opt, elem_bytes(delta_dtype))), MDZ_EINVAL,
              "residual_rmsnorm_i8: a buffer is not aligned to its elements");
  hipStream_t st = (hipStream_t)stream;
  if (!delta_opt || delta_dtype == MDZ_FP32)
    MDZ_WITH_ELEM(dtype, return launch_rows_i8<E>(NormRows<E, float>{x, (const float*)delta_opt, (const E*)gain, x_out_opt, d, eps}, rows, d,
                                                  codes, scales, values_opt, st));
  MDZ_WITH_ELEM(dtype, return launch_rows_i8<E>(NormRows<E, E>{x, (const E*)delta_opt, (const E*)gain, x_out_opt, d, eps}, rows, d, codes,
                                                scales, values_opt, st));
}

#pragma GCC visibility pop
}  // extern "C"
