// Matrices in 4 bits: packing, how a product is cut, and the C entries.  The kernel stands in gemm_i4.h.
#include "i4.h"

namespace mdz {

// ---- packing (once per matrix) -----------------------------------------------------------------------
// A thread makes one word (eight codes of a row); the thread of a group's first word writes its scale and zero point.  Source: codes, scales and zero
// points as they are, or (src) a matrix to be quantised, whose group each of its threads goes over.
struct I4Source {
  const void* src;
  const uint8_t* codes;
  const void* scales;
  const uint8_t* zeros;
};
// Codes are bound by memory: 128000 x 4096 in 210 us, 3.8 TB/s in and out, with 8-byte loads and 32-bit divisions (988 us with single bytes and 64-bit ones).  Quantising, once
// when a model is loaded, is bound by the threads' way over their group by single elements: 128000 x 4096 of bf16 in groups of 128 4.8 ms, 4096 x 4096 148 us.
template <typename E>
__global__ void __launch_bounds__(256) pack_i4_kernel(I4Source s, int64_t n_rows, int k, int group, bool with_zeros, uint32_t* __restrict__ codes,
                                                      E* __restrict__ scales, uint8_t* __restrict__ zeros, uint32_t blocks, int64_t words) {
  const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (w >= words) return;
  const uint32_t at = (uint32_t)(w >> 8), tile = at / blocks, block = at - tile * blocks;  // (words are fewer than 2^32)
  const int lane = (int)(w >> 2) & 63, r = lane & 15, in_block = (int)(w & 3) * 32 + (lane >> 4) * 8, log_group = 31 - __clz(group);
  const int k0 = (int)block * kI4Block + in_block, groups = (k + group - 1) >> log_group, g = k0 >> log_group;
  const int64_t n = (int64_t)tile * 16 + r;
  float scale = 0.f;
  int zero = 8, q[8] = {8, 8, 8, 8, 8, 8, 8, 8};
  if (n < n_rows && g < groups) {
    if (s.src) {
      const E* row = reinterpret_cast<const E*>(s.src) + n * k;
      const int end = (int)min((int64_t)(g + 1) * group, (int64_t)k);
      float lo = 0.f, hi = 0.f;
      bool bad = false;
      for (int i = g * group; i < end; ++i) {
        const float v = to_float(row[i]);
        bad |= !(fabsf(v) < INFINITY);
        lo = fminf(lo, v), hi = fmaxf(hi, v);
      }
      // the scale as it will be read: rounded to the storage type
      scale = to_float(from_float<E>(with_zeros ? hi / 15.f - lo / 15.f : fmaxf(hi, fabsf(lo)) / 7.f));
      if (bad) {
        scale = __uint_as_float(0x7FC00000u);
      } else if (scale > 0.f) {
        if (with_zeros) zero = (int)fminf(fmaxf(rintf(-lo / scale), 0.f), 15.f);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          q[e] = k0 + e < k ? (int)fminf(fmaxf(rintf(to_float(row[k0 + e]) / scale) + (float)zero, 0.f), 15.f) : zero;
      }
    } else {
      scale = to_float(reinterpret_cast<const E*>(s.scales)[n * groups + g]);
      if (with_zeros) zero = s.zeros[n * groups + g] & 15;
      const uint8_t* const c = s.codes + n * k + k0;
      if (k0 + 8 <= k) {
        typedef uint64_t Any8 __attribute__((aligned(1)));
        const uint64_t eight = *reinterpret_cast<const Any8*>(c);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = (int)(eight >> (8 * e)) & 15;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = k0 + e < k ? c[e] & 15 : zero;
      }
    }
  }
  uint32_t word = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) word |= (uint32_t)q[e] << (4 * i4_field(e));
  codes[w] = word << kI4Rotation<E> | word >> (32 - kI4Rotation<E>);
  if (in_block % group == 0) {
    const int64_t to = ((int64_t)at * 16 + r) * (kI4Block >> log_group) + (in_block >> log_group);
    scales[to] = from_float<E>(scale);
    if (with_zeros) zeros[to] = (uint8_t)zero;
  }
}

static int check_sizes_i4(const char* what, int64_t n_rows, int64_t k, int group, int zeros) {
  MDZ_REQUIRE(n_rows > 0 && k > 0, MDZ_EINVAL, "%s: sizes must be positive", what);
  MDZ_REQUIRE(i4_group_ok(group) && (zeros == 0 || zeros == 1), MDZ_EINVAL, "%s: groups of 32, 64 or 128 features (%d), zeros 0 or 1 (%d)", what, group, zeros);
  MDZ_REQUIRE(k <= kI4MaxK && n_rows <= INT32_MAX - kI4TileRows, MDZ_EUNSUPPORTED, "%s: [%lld,%lld]: up to %d input features and 2^31 rows", what,
              (long long)n_rows, (long long)k, kI4MaxK);
  return MDZ_OK;
}

static int pack_i4(int dtype, const I4Source& s, int64_t n_rows, int64_t k, int group, int zeros, void* dst, int64_t dst_rows, int64_t tile_offset,
                   void* stream) {
  MDZ_REQUIRE(is_16bit(dtype), dtype_ok(dtype) ? MDZ_EUNSUPPORTED : MDZ_EINVAL, "pack i4: dtype %d: bf16 or fp16", dtype);
  MDZ_REQUIRE((s.src || (s.codes && s.scales)) && dst, MDZ_EINVAL, "pack i4: NULL pointer");
  const int rc = check_sizes_i4("pack i4", dst_rows, k, group, zeros);
  if (rc) return rc;
  MDZ_REQUIRE(n_rows > 0 && dst_rows >= n_rows && tile_offset >= 0, MDZ_EINVAL, "pack i4: bad sizes");
  MDZ_REQUIRE((reinterpret_cast<uintptr_t>(dst) & 15) == 0, MDZ_EINVAL, "pack i4: the packed matrix must start on 16 bytes");
  MDZ_REQUIRE((reinterpret_cast<uintptr_t>(s.src) | reinterpret_cast<uintptr_t>(s.scales)) % 2 == 0, MDZ_EINVAL,
              "pack i4: a buffer is not aligned to its elements");
  const int64_t tiles = i4_tiles(n_rows), all = i4_tiles(dst_rows);
  MDZ_REQUIRE(tile_offset <= all && tile_offset + tiles <= all, MDZ_ESHAPE, "pack i4: %lld rows at tile %lld exceed dst_rows %lld", (long long)n_rows,
              (long long)tile_offset, (long long)dst_rows);
  MDZ_REQUIRE(n_rows % kI4TileRows == 0 || tile_offset + tiles == all, MDZ_ESHAPE,
              "pack i4: n_rows %lld is not a multiple of the tile height %d and this is not the last matrix", (long long)n_rows, kI4TileRows);
  const int64_t blocks = i4_blocks(k), words = tiles * blocks * 256, first = tile_offset * blocks, groups = kI4Block / group;
  MDZ_REQUIRE(words <= (int64_t)UINT32_MAX - 255, MDZ_EUNSUPPORTED, "pack i4: [%lld,%lld] is more than one launch takes", (long long)n_rows, (long long)k);
  char* const to = (char*)dst;
  hipStream_t st = (hipStream_t)stream;
  ProfScope prof_(PROF_MISC, st);
  MDZ_WITH_ELEM16(dtype, (pack_i4_kernel<E><<<(unsigned)((words + 255) / 256), 256, 0, st>>>(
                             s, n_rows, (int)k, group, zeros != 0, (uint32_t*)(to + first * 1024), (E*)(to + i4_scales_offset(dst_rows, k) + first * 32 * groups),
                             (uint8_t*)(to + i4_zeros_offset(dst_rows, k, group) + first * 16 * groups), (uint32_t)blocks, words)));
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

// ---- products ----------------------------------------------------------------------------------------
// Up to 16 rows the weights are the stream and each workgroup of the kernel of few rows takes one column tile (pair) until every CU has one, with eight waves on
// its features, then two and four with four waves.  (us at 1 row, one / two / four tiles: 4096 x 4096 5.2 / 6.0 / 8.3; 12288 x 4096 11.8 / 9.5 / 9.0;
// 22016 x 4096 19.5 / 12.8 / 13.5; 128000 x 4096 72.6 / 59.8 / 56.7; 16 rows 12288 x 4096 17.1 / 11.5 / 10.1; gated 688 pairs, one / two: 12.7 / 14.4 at 1 row,
// 17.4 / 16.1 at 16.)  In groups of 32 four tiles do not fit the registers (12288 x 4096 at 1 row, two / four: 11.3 / 19.9; with zero points in bf16
// two tiles with eight / four waves: 17.1 / 20.8).
// Beyond, the cut of the least modelled time: rounds of workgroups over the chip x turns of a workgroup x a turn's us (kI4Cuts).
constexpr int kMaxGridY = 65535;
static I4Plan plan_i4(int M, int N, int K, int kind, bool gated) {
  const int64_t tiles = i4_tiles(N), blocks = i4_blocks(K), cus = num_cus();
  if (M <= 16) {
    const int xr = M <= 4 ? 1 : M <= 8 ? 2 : 4;
    const bool of_32 = kind == 2 || kind == 5 || kind == 7;
    const I4Plan two{1, 2, kind == 5 ? 8 : 4, xr}, four{1, 4, 4, xr};
    if (gated) return tiles <= cus ? I4Plan{1, 2, 8, xr} : of_32 || (tiles <= 4 * cus && xr < 4) ? two : four;
    return tiles <= cus ? I4Plan{1, 1, 8, xr} : of_32 || tiles <= 2 * cus ? two : four;
  }
  I4Plan best{};
  float least = INFINITY;
  for (const I4Cut& c : kI4Cuts) {
    const int wide = gated ? c.gate_tiles : c.tiles;
    if (M < c.least_rows || M > c.most_rows || wide == 0 || c.us[kind] == 0.f) continue;
    if (c.plan.xr != 0 && (M + c.rows - 1) / c.rows > kMaxGridY) continue;  // (its rows are the grid's second axis)
    const int64_t wgs = ((int64_t)(M + c.rows - 1) / c.rows) * ((tiles + wide - 1) / wide), at_once = c.us_two[kind] > 0.f ? 2 * cus : cus;
    const int64_t full = wgs / at_once, rest = wgs % at_once;
    const float us_full = at_once > cus ? c.us_two[kind] : c.us[kind], us_rest = rest > cus ? us_full : rest > 0 ? c.us[kind] : 0.f;
    const float us = ((float)full * us_full + us_rest) * (float)((blocks + c.features - 1) / c.features);
    if (us < least) best = c.plan, least = us;
  }
  return best;
}

// Rows that do not start on 16 bytes, again 16 bytes apart and padded with zeros to whole blocks: a thread makes eight features.
__global__ void __launch_bounds__(256) align_rows_i4_kernel(const uint16_t* __restrict__ x, int K, u32x4_t* __restrict__ out, int64_t chunks, int per_row) {
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (q >= chunks) return;
  const int64_t row = q / per_row;
  const int k = (int)(q - row * per_row) * 8;
  u32x4_t v{0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (k + e < K) v[e >> 1] |= (uint32_t)x[row * K + k + e] << (16 * (e & 1));
  out[q] = v;
}
// scratch for them
static int64_t aligned_bytes_i4(int M, int K) { return M <= 16 ? 0 : (int64_t)M * i4_blocks(K) * kI4Block * 2; }

static int check_product_i4(const char* what, int M, int N, int K) {
  MDZ_REQUIRE(M >= 0 && N > 0 && K > 0, MDZ_EINVAL, "%s: [%d,%d] x [%d,%d]", what, M, K, N, K);
  MDZ_REQUIRE(K <= kI4MaxK && M <= 1 << 30 && N <= 1 << 30 && (int64_t)M * N < (int64_t)1 << 40, MDZ_EUNSUPPORTED,
              "%s: [%d,%d] x [%d,%d]: up to %d input features, 2^30 rows and columns and 2^40 outputs", what, M, K, N, K, kI4MaxK);
  return MDZ_OK;
}

static int product_i4(const char* what, int dtype, const void* x, const void* packed, const void* second, int M, int N, int K, int group, int zeros,
                      int out_dtype, void* y, void* ws, int64_t ws_bytes, void* stream) {
  MDZ_REQUIRE(is_16bit(dtype), dtype_ok(dtype) ? MDZ_EUNSUPPORTED : MDZ_EINVAL, "%s: dtype %d: bf16 or fp16", what, dtype);
  MDZ_REQUIRE(dtype_ok(out_dtype), MDZ_EINVAL, "%s: bad dtype %d", what, out_dtype);
  MDZ_REQUIRE(i4_group_ok(group) && (zeros == 0 || zeros == 1), MDZ_EINVAL, "%s: groups of 32, 64 or 128 features (%d), zeros 0 or 1 (%d)", what, group, zeros);
  const int rc = check_product_i4(what, M, N, K);
  if (rc) return rc;
  if (M == 0) return MDZ_OK;
  MDZ_REQUIRE(x && packed && y, MDZ_EINVAL, "%s: NULL pointer", what);
  MDZ_REQUIRE(((reinterpret_cast<uintptr_t>(packed) | reinterpret_cast<uintptr_t>(second)) & 15) == 0, MDZ_EINVAL,
              "%s: a packed matrix must start on 16 bytes", what);
  MDZ_REQUIRE(reinterpret_cast<uintptr_t>(x) % 2 == 0 && reinterpret_cast<uintptr_t>(y) % elem_bytes(out_dtype) == 0, MDZ_EINVAL,
              "%s: a buffer is not aligned to its elements", what);
  I4Product p{};
  p.X = x, p.w[0] = i4_matrix(packed, N, K, group), p.w[1] = i4_matrix(second ? second : packed, N, K, group), p.Y = y;
  p.M = M, p.N = N, p.K = K, p.out_dtype = out_dtype, p.n_tiles = (int)i4_tiles(N), p.n_blocks = (int)i4_blocks(K);
  const int64_t need = aligned_bytes_i4(M, K);
  MDZ_REQUIRE(ws_bytes >= need && (ws || need == 0), MDZ_EWORKSPACE, "%s: workspace %lld < %lld bytes", what, (long long)ws_bytes, (long long)need);
  MDZ_REQUIRE(need == 0 || (reinterpret_cast<uintptr_t>(ws) & 15) == 0, MDZ_EINVAL, "%s: the workspace must start on 16 bytes", what);
  const I4Plan plan = plan_i4(M, N, K, i4_kind(dtype == MDZ_FP16, kI4Block / group, zeros != 0), second != nullptr);
  hipStream_t st = (hipStream_t)stream;
  const bool z = zeros != 0, gated = second != nullptr;
  p.ldx = (int64_t)K * 2;
  if (plan.xr == 0 && (K % 8 != 0 || reinterpret_cast<uintptr_t>(x) % 16 != 0)) {  // loads to LDS take 16 bytes from addresses of 16
    const int64_t chunks = need / 16;
    MDZ_REQUIRE(chunks <= (int64_t)UINT32_MAX - 255, MDZ_EUNSUPPORTED, "%s: %d unaligned rows are more than one launch takes", what, M);
    launch_timed(PROF_GEMM_I4, align_rows_i4_kernel, (unsigned)((chunks + 255) / 256), 256, 0, st, (const uint16_t*)x, K, (u32x4_t*)ws, chunks,
                 p.n_blocks * (kI4Block / 8));
    MDZ_LAUNCH_CHECK();
    p.X = ws, p.K = p.n_blocks * kI4Block, p.ldx = (int64_t)p.K * 2;
  }
  MDZ_WITH_ELEM16(dtype, return (group == 128 ? launch_i4<E, 1>(p, z, gated, plan, st) : group == 64 ? launch_i4<E, 2>(p, z, gated, plan, st)
                                                                                                  : launch_i4<E, 4>(p, z, gated, plan, st)));
}

}  // namespace mdz

using namespace mdz;

extern "C" {
#pragma GCC visibility push(default)

int64_t medusa_packed_i4_bytes(int64_t n_rows, int64_t k, int group, int zeros) {
  const int rc = check_sizes_i4("packed_i4_bytes", n_rows, k, group, zeros);
  return rc ? rc : i4_packed_bytes(n_rows, k, group, zeros != 0);
}

int medusa_pack_weight_i4(int dtype, const void* src, int64_t n_rows, int64_t k, int group, int zeros, void* dst, int64_t dst_rows, int64_t tile_offset,
                          void* stream) {
  return pack_i4(dtype, I4Source{src, nullptr, nullptr, nullptr}, n_rows, k, group, zeros, dst, dst_rows, tile_offset, stream);
}

int medusa_pack_codes_i4(int dtype, const uint8_t* codes, const void* scales, const uint8_t* zeros_opt, int64_t n_rows, int64_t k, int group, void* dst,
                         int64_t dst_rows, int64_t tile_offset, void* stream) {
  return pack_i4(dtype, I4Source{nullptr, codes, scales, zeros_opt}, n_rows, k, group, zeros_opt != nullptr, dst, dst_rows, tile_offset, stream);
}

int64_t medusa_linear_i4_workspace_bytes(int M, int N, int K) {
  const int rc = check_product_i4("linear_i4", M, N, K);
  return rc ? rc : aligned_bytes_i4(M, K);
}

int64_t medusa_swiglu_i4_workspace_bytes(int M, int ffn, int K) {
  const int rc = check_product_i4("swiglu_i4", M, ffn, K);
  return rc ? rc : aligned_bytes_i4(M, K);
}

int medusa_linear_i4(int dtype, const void* x, const void* packed, int M, int N, int K, int group, int zeros, int out_dtype, void* y, void* ws,
                     int64_t ws_bytes, void* stream) {
  return product_i4("linear_i4", dtype, x, packed, nullptr, M, N, K, group, zeros, out_dtype, y, ws, ws_bytes, stream);
}

int medusa_swiglu_i4(int dtype, const void* x, const void* gate_packed, const void* up_packed, int M, int ffn, int K, int group, int zeros, void* y, void* ws,
                     int64_t ws_bytes, void* stream) {
  MDZ_REQUIRE(gate_packed && up_packed, MDZ_EINVAL, "swiglu_i4: NULL pointer");
  return product_i4("swiglu_i4", dtype, x, gate_packed, up_packed, M, ffn, K, group, zeros, dtype, y, ws, ws_bytes, stream);
}

#pragma GCC visibility pop
}  // extern "C"
