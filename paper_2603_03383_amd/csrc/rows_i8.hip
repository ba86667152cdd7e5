// Rows in 8 bits with one scale each: the residual's addition and RMSNorm, SwiGLU, plain rows, and the packing of 8-bit weights.
//
// A row is one workgroup's: its elements are read once, stay in registers while max|t| (and the norm's sum of squares) go around the
// workgroup in a single exchange, and leave as codes.  The norm needs no second exchange for its factor, because 1 / rms is positive:
// the codes of x' * gain / rms are those of x' * gain, and the factor goes into the scale.  So the codes do not depend on the order of any sum.
// What bounds it: up to a row per CU the latency of one load, one exchange and one store (a launch of 4.0-4.8 us, 64 rows of 4096 like
// one); beyond, memory.  By the stamps of a launch: norm 1024 x 5120 (16-bit update, 16-bit values written too) 13.1 us = 5.2 TB/s, 4096 x 8192
// 78 us = 5.6 TB/s, SwiGLU 1024 x 12800 20.2 us = 4.5 TB/s, 2048 x 11008 33.5 us = 4.7 TB/s, against 4.9 TB/s of a large copy.  (In a row of
// calls, where launches overlap at their ends, the first takes 12.4 us a call and the third 16.9.)
#include "i8.h"

namespace mdz {

__device__ inline uint32_t max_u(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Over a wave by lane permutations (no trip through LDS), the result in every lane: rows of 16 lanes first, then across them.
template <int CTRL, int ROWS>
__device__ inline uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <typename Op>
__device__ inline uint32_t wave_reduce(uint32_t v, Op op) {  // zero bits are neutral
  v = op(v, dpp<0x111, 0xf>(v));  // row_shr 1, 2, 4, 8: lane 15 of a row has the row
  v = op(v, dpp<0x112, 0xf>(v));
  v = op(v, dpp<0x114, 0xf>(v));
  v = op(v, dpp<0x118, 0xf>(v));
  v = op(v, dpp<0x142, 0xa>(v));  // lane 15 of a row to the next row (1 and 3), lane 31 to the rows 2 and 3
  v = op(v, dpp<0x143, 0xc>(v));
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ inline float wave_sum(float v) {
  return __uint_as_float(wave_reduce(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ inline uint32_t wave_max(uint32_t v) { return wave_reduce(v, max_u); }

// A row's statistics over the workgroup: max|t| (bits) and the sum of squares, in one exchange.
__device__ inline void row_statistics(uint32_t& amax, float& squares) {
  __shared__ uint32_t wave_amax[16];
  __shared__ float wave_squares[16];
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  amax = wave_max(amax), squares = wave_sum(squares);
  if ((threadIdx.x & 63) == 0) wave_amax[wave] = amax, wave_squares[wave] = squares;
  __syncthreads();
  amax = 0, squares = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    const uint32_t a = wave_amax[w];
    const float q = wave_squares[w];
    amax = w < waves ? max_u(amax, a) : amax, squares += w < waves ? q : 0.f;
  }
}

// W elements as one load or store of any alignment
template <int BYTES>
struct Piece;
template <>
struct Piece<4> {
  typedef uint32_t Bits;
  typedef Bits Any __attribute__((aligned(1)));
};
template <>
struct Piece<8> {
  typedef uint32_t Bits __attribute__((ext_vector_type(2)));
  typedef Bits Any __attribute__((aligned(1)));
};
template <>
struct Piece<16> {
  typedef u32x4_t Bits;
  typedef Bits Any __attribute__((aligned(1)));
};
template <typename E, int W>
struct Elems {
  E v[W];
};
// W consecutive elements of a row.  TAIL (the row's width is no multiple of W): near its end `n` < W are there, the others come as zero.
template <bool TAIL, int W, typename E>
__device__ inline Elems<E, W> fetch(const E* src, int n) {
  typedef Piece<W * sizeof(E)> P;
  typedef Elems<E, W> Some;
  Some s;
  if (!TAIL || n >= W) {
    const typename P::Bits bits = *reinterpret_cast<const typename P::Any*>(src);
    s = __builtin_bit_cast(Some, bits);
  } else {
#pragma unroll
    for (int e = 0; e < W; ++e) s.v[e] = e < n ? src[e] : E{};
  }
  return s;
}
template <bool TAIL, int W, typename E>
__device__ inline void put(E* dst, int n, const Elems<E, W>& s) {
  typedef Piece<W * sizeof(E)> P;
  if (!TAIL || n >= W) {
    *reinterpret_cast<typename P::Any*>(dst) = __builtin_bit_cast(typename P::Bits, s);
  } else {
#pragma unroll
    for (int e = 0; e < W; ++e)
      if (e < n) dst[e] = s.v[e];
  }
}

// Where a kernel's rows come from: `load` requests kW elements of row r from element i on, `n` of them inside the row, and `values` makes
// them numbers.
template <typename E>
struct PlainRows {
  static constexpr int kW = 16 / sizeof(E);
  struct Raw {
    Elems<E, kW> x;
  };
  const E* src;
  int d;
  template <bool TAIL>
  __device__ inline void load(int64_t r, int i, int n, Raw& raw) const {
    raw.x = fetch<TAIL, kW>(src + r * d + i, n);
  }
  template <bool TAIL>
  __device__ inline void values(int64_t, int, int, const Raw& raw, float (&t)[kW], float&) const {
#pragma unroll
    for (int e = 0; e < kW; ++e) t[e] = to_float(raw.x.v[e]);
  }
  __device__ inline float factor(float) const { return 1.f; }
  __device__ inline void second_reading() {}
};
// 1 / (1 + e^-g): the exponential's argument in two parts, so that its rounding does not grow with g; one unit in the last place each for
// the exponential and the reciprocal.  (Where the argument's high part is infinite the low part is not a number; from 2^127 on the
// sigmoid is below fp32's normal range, and below 2^-127 it is 1.)
__device__ inline float sigmoid_i8(float g) {
  constexpr float kLog2e = 1.44269504f, kLow = 1.92596303e-8f;  // log2(e) = their sum
  const float hi = -g * kLog2e;
  const float lo = fmaf(-g, kLog2e, -hi) - g * kLow;
  const float e = fast_exp2(hi);
  return __builtin_amdgcn_rcpf(1.f + (fabsf(hi) < 127.f ? fmaf(e, lo * 0.693147181f, e) : e));
}
template <typename E>
struct SwigluRows {
  static constexpr int kW = 16 / sizeof(E);
  struct Raw {
    Elems<E, kW> gate, up;
  };
  const E* gate_up;
  int d;
  template <bool TAIL>
  __device__ inline void load(int64_t r, int i, int n, Raw& raw) const {
    raw.gate = fetch<TAIL, kW>(gate_up + r * 2 * d + i, n);
    raw.up = fetch<TAIL, kW>(gate_up + r * 2 * d + d + i, n);
  }
  template <bool TAIL>
  __device__ inline void values(int64_t, int, int, const Raw& raw, float (&t)[kW], float&) const {
#pragma unroll
    for (int e = 0; e < kW; ++e) {
      const float g = to_float(raw.gate.v[e]);
      t[e] = g * sigmoid_i8(g) * to_float(raw.up.v[e]);
    }
  }
  __device__ inline float factor(float) const { return 1.f; }
  __device__ inline void second_reading() {}
};
// x' = x + delta; the codes are those of x' * gain, because the norm's factor is positive and cancels; it goes into the scale
template <typename E, typename D>
struct NormRows {
  static constexpr int kW = 4;
  struct Raw {
    Elems<float, kW> x;
    Elems<D, kW> delta;
    Elems<E, kW> gain;
  };
  const float* x;
  const D* delta;
  const E* gain;
  float* x_out;
  int d;
  float eps;
  template <bool TAIL>
  __device__ inline void load(int64_t r, int i, int n, Raw& raw) const {
    raw.x = fetch<TAIL, kW>(x + r * d + i, n);
    if (delta) raw.delta = fetch<TAIL, kW>(delta + r * d + i, n);
    raw.gain = fetch<TAIL, kW>(gain + i, n);
  }
  template <bool TAIL>
  __device__ inline void values(int64_t r, int i, int n, const Raw& raw, float (&t)[kW], float& squares) const {
    Elems<float, kW> sum = raw.x;
    if (delta) {
#pragma unroll
      for (int e = 0; e < kW; ++e) sum.v[e] += to_float(raw.delta.v[e]);
    }
    if (x_out && n > 0) put<TAIL, kW>(x_out + r * d + i, n, sum);
#pragma unroll
    for (int e = 0; e < kW; ++e) {
      squares += n > 0 ? sum.v[e] * sum.v[e] : 0.f;
      t[e] = sum.v[e] * to_float(raw.gain.v[e]);
    }
  }
  __device__ inline float factor(float squares) const { return 1.f / sqrtf(squares / (float)d + eps); }
  // a thread reads again what it wrote itself: x_out may be x, which holds the sum by then
  __device__ inline void second_reading() {
    if (x_out) x = x_out, delta = nullptr, x_out = nullptr;
  }
};

// The same with the update still in parts: finished here as the product's own second launch would.  x' and the codes are bit for bit those of the
// product and NormRows; the sum of squares is one fused operation per element there where the compiler makes it one, two roundings here, so scales can
// differ in their last bits.
template <typename E>
struct NormOfSumsRows {
  static constexpr int kW = 4;
  typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
  struct Raw {
    Elems<float, kW> x, sw;
    Elems<E, kW> gain;
    i32x4 part[kI8MaxParts];
    float sx;
  };
  float* x;
  I8Sums sums;
  const E* gain;
  int d;
  float eps;
  template <bool TAIL>
  __device__ inline void load(int64_t r, int i, int n, Raw& raw) const {
    raw.x = fetch<TAIL, kW>(x + r * d + i, n);
#pragma unroll
    for (int s = 0; s < kI8MaxParts; ++s)
      if (s < sums.n) raw.part[s] = *reinterpret_cast<const i32x4*>(sums.parts + s * sums.stride + r * sums.ld + i);
    raw.sx = sums.sx[r];
    raw.sw = fetch<TAIL, kW>(sums.sw + i, n);
    raw.gain = fetch<TAIL, kW>(gain + i, n);
  }
  template <bool TAIL>
  __device__ inline void values(int64_t r, int i, int n, const Raw& raw, float (&t)[kW], float& squares) const {
#pragma clang fp contract(off)  // every rounding of x' as where the product is stored in between
    i32x4 sum = raw.part[0];
#pragma unroll
    for (int s = 1; s < kI8MaxParts; ++s)
      if (s < sums.n) sum += raw.part[s];
    Elems<float, kW> y;
#pragma unroll
    for (int e = 0; e < kW; ++e) {
      y.v[e] = raw.x.v[e] + (float)sum[e] * (raw.sx * raw.sw.v[e]);
      squares += n > 0 ? y.v[e] * y.v[e] : 0.f;
      t[e] = y.v[e] * to_float(raw.gain.v[e]);
    }
    if (n > 0) put<TAIL, kW>(x + r * d + i, n, y);
  }
  __device__ inline float factor(float squares) const { return 1.f / sqrtf(squares / (float)d + eps); }
};

// codes of t and what they stand for, W at a time
template <bool TAIL, typename E, int W>
__device__ inline void put_codes(const I8Quantiser& q, const float (&t)[W], int n, float scale, int8_t* codes, E* values) {
  Elems<int8_t, W> c;
  Elems<E, W> v;
  float code[W];
  q.round(t, code);
#pragma unroll
  for (int e = 0; e < W; ++e) {
    c.v[e] = (int8_t)(int)code[e];
    v.v[e] = from_float<E>(code[e] * scale);
  }
  put<TAIL, W>(codes, n, c);
  if (values) put<TAIL, W>(values, n, v);
}

// One workgroup per row, whose elements stay in registers from the statistics to the codes: a thread has NV pieces of kW.
template <typename Rows, typename E, int NV, bool TAIL>
__global__ void __launch_bounds__(1024) rows_i8_kernel(Rows in, int d, int8_t* codes, float* scales, E* values) {
  constexpr int W = Rows::kW;
  const int64_t r = blockIdx.x;
  typename Rows::Raw raw[NV];
  float t[NV][W], squares = 0.f;
  uint32_t amax = 0;
#pragma unroll
  for (int k = 0; k < NV; ++k) {  // everything is requested before the first of it is used; beyond the row its start again
    const int i = (threadIdx.x + k * blockDim.x) * W;
    in.template load<TAIL>(r, i < d ? i : 0, TAIL ? d - i : W, raw[k]);
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = (threadIdx.x + k * blockDim.x) * W;
    in.template values<TAIL>(r, i, d - i, raw[k], t[k], squares);
#pragma unroll
    for (int e = 0; e < W; ++e) amax = max_u(amax, i < d ? abs_bits(t[k][e]) : 0u);
  }
  row_statistics(amax, squares);
  const I8Quantiser q(amax);
  const float scale = q.scale_times(in.factor(squares));
  if (threadIdx.x == 0) scales[r] = scale;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = (threadIdx.x + k * blockDim.x) * W;
    if (i < d) put_codes<TAIL, E, W>(q, t[k], d - i, scale, codes + r * d + i, values ? values + r * d + i : nullptr);
  }
}

// Rows longer than the registers of a workgroup: read twice.
template <typename Rows, typename E>
__global__ void __launch_bounds__(1024) rows_i8_long_kernel(Rows in, int d, int8_t* codes, float* scales, E* values) {
  constexpr int W = Rows::kW;
  const int64_t r = blockIdx.x;
  typename Rows::Raw raw;
  float t[W], squares = 0.f;
  uint32_t amax = 0;
  for (int i = threadIdx.x * W; i < d; i += 1024 * W) {
    in.template load<true>(r, i, d - i, raw);
    in.template values<true>(r, i, d - i, raw, t, squares);
#pragma unroll
    for (int e = 0; e < W; ++e) amax = max_u(amax, abs_bits(t[e]));
  }
  row_statistics(amax, squares);
  const I8Quantiser q(amax);
  const float scale = q.scale_times(in.factor(squares));
  if (threadIdx.x == 0) scales[r] = scale;
  in.second_reading();
  for (int i = threadIdx.x * W; i < d; i += 1024 * W) {
    float unused = 0.f;
    in.template load<true>(r, i, d - i, raw);
    in.template values<true>(r, i, d - i, raw, t, unused);
    put_codes<true, E, W>(q, t, d - i, scale, codes + r * d + i, values ? values + r * d + i : nullptr);
  }
}

template <typename E, bool TAIL, typename Rows>
static auto rows_i8_variant(const Rows&, int nv) {
  return nv == 1 ? rows_i8_kernel<Rows, E, 1, TAIL> : nv == 2 ? rows_i8_kernel<Rows, E, 2, TAIL> : rows_i8_kernel<Rows, E, 4, TAIL>;
}
// ANY: any width; else whole pieces that fit the registers of a workgroup
template <typename E, bool ANY, typename Rows>
static int launch_rows_i8(const Rows& in, int rows, int d, int8_t* codes, float* scales, void* values, hipStream_t st) {
  if (rows == 0) return MDZ_OK;
  const int pieces = (d + Rows::kW - 1) / Rows::kW;
  // Up to a row per CU a row's time is the latency of one thread's chain, so a thread takes as little as it can; with more rows, small
  // workgroups leave a CU no idle while one of them starts or ends.  us with up to 1024 / 256 threads before a thread takes more:
  // SwiGLU 64 x 11008 5.1 / 6.1; norm 1024 x 5120 15.3 / 13.1, 1024 x 4096 13.6 / 11.5, SwiGLU 1024 x 12800 21.9 / 20.2.
  const int most = rows <= num_cus() ? 1024 : 256;
  const int nv = pieces <= most ? 1 : pieces <= 2 * most ? 2 : 4;
  int threads = ((pieces + nv - 1) / nv + 63) / 64 * 64;
  auto kernel = rows_i8_variant<E, false>(in, nv);
  if constexpr (ANY) {
    if (d % Rows::kW) kernel = rows_i8_variant<E, true>(in, nv);
    if (pieces > 4096) kernel = rows_i8_long_kernel<Rows, E>, threads = 1024;
  }
  MDZ_REQUIRE(i8_launchable(rows, threads), MDZ_EUNSUPPORTED, "rows i8: %d rows of %d are more than one launch takes", rows, d);
  launch_timed(PROF_ROWS_I8, kernel, rows, threads, 0, st, in, d, codes, scales, (E*)values);
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

int launch_residual_rmsnorm_i8(int dtype, float* x, const float* delta, const I8Sums& sums, const void* gain, float eps, int rows, int d,
                               int8_t* codes, float* scales, hipStream_t st) {
  if (sums.n == 0)
    return medusa_residual_rmsnorm_i8(dtype, x, delta, MDZ_FP32, gain, eps, rows, d, x, codes, scales, nullptr, st);
  MDZ_REQUIRE(d % 4 == 0 && d <= kI8MaxPartsWidth && sums.n <= kI8MaxParts, MDZ_EUNSUPPORTED, "norm i8: width %d, %d parts", d, sums.n);
  MDZ_WITH_ELEM16(dtype, return (launch_rows_i8<E, false>(NormOfSumsRows<E>{x, sums, (const E*)gain, d, eps}, rows, d, codes, scales, nullptr, st)));
}

// One workgroup per row of the padded matrix: codes and scale of a source row, zeros for a row of the padding.
template <typename E>
__global__ void __launch_bounds__(256) pack_weight_i8_kernel(const E* src, int64_t n_rows, int64_t k, uint8_t* dst, int64_t kp,
                                                             int64_t first_row, float* scales) {
  const int64_t n = blockIdx.x, row = first_row + n;
  uint32_t amax = 0;
  float unused = 0.f;
  if (n < n_rows)
    for (int64_t i = threadIdx.x; i < k; i += 256) amax = max_u(amax, abs_bits(to_float(src[n * k + i])));
  row_statistics(amax, unused);
  const I8Quantiser q(amax);
  if (threadIdx.x == 0) scales[row] = n < n_rows ? q.scale : 0.f;
  for (int64_t i = threadIdx.x; i < kp; i += 256) {
    float t[1] = {n < n_rows && i < k ? to_float(src[n * k + i]) : 0.f}, c[1];
    q.round(t, c);
    dst[i8_index(row, i, kp)] = (uint8_t)(int8_t)(int)c[0];
  }
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
  MDZ_REQUIRE(i8_launchable(i8_padded_rows(n_rows), 256), MDZ_EUNSUPPORTED, "pack i8: %lld rows are more than one launch takes", (long long)n_rows);
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
  MDZ_WITH_ELEM(dtype, return (launch_rows_i8<E, true>(PlainRows<E>{(const E*)src, d}, rows, d, codes, scales, values_opt, (hipStream_t)stream)));
}

int medusa_swiglu_i8(int dtype, const void* gate_up, int rows, int ffn, int8_t* codes, float* scales, void* values_opt, void* stream) {
  int rc = check_rows_i8("swiglu_i8", dtype, gate_up, elem_bytes(dtype), rows, ffn, codes, scales, values_opt);
  if (rc) return rc;
  MDZ_WITH_ELEM(dtype, return (launch_rows_i8<E, true>(SwigluRows<E>{(const E*)gate_up, ffn}, rows, ffn, codes, scales, values_opt,
                                                       (hipStream_t)stream)));
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
    MDZ_WITH_ELEM(dtype, return (launch_rows_i8<E, true>(NormRows<E, float>{x, (const float*)delta_opt, (const E*)gain, x_out_opt, d, eps},
                                                         rows, d, codes, scales, values_opt, st)));
  MDZ_WITH_ELEM(dtype, return (launch_rows_i8<E, true>(NormRows<E, E>{x, (const E*)delta_opt, (const E*)gain, x_out_opt, d, eps}, rows, d,
                                                     codes, scales, values_opt, st)));
}

#pragma GCC visibility pop
}  // extern "C"
