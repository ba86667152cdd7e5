// Product of rows in 8 bits with packed 8-bit weights: y[m][n] = sx[m] * sw[n] * sum_k cx[m][k] * cw[n][k], sums in 32-bit integers.  Here:
// which kernel a product takes, the kernel of few rows, and the C entry.
#include "gemm_i8.h"

namespace mdz {

// 16 codes of a row of K from feature k on (any alignment); features beyond K come as zeros
__device__ inline i32x4 load_codes(const int8_t* row, int k, int K) {
  typedef i32x4 i32x4_any __attribute__((aligned(1)));
  if (k + 16 <= K) return *reinterpret_cast<const i32x4_any*>(row + k);
  i32x4 v{0, 0, 0, 0};
  for (int j = 0; j < K - k; ++j) v[j >> 2] |= (int32_t)(uint8_t)row[k + j] << (8 * (j & 3));
  return v;
}

// Few rows: W is the stream.  A workgroup of NW waves makes MT 16-row x NT 16-column tiles; the waves share out the features, so each reads
// contiguous memory, W in whole kilobytes (non-temporal: each is read once) and the rows, which all workgroups share, beside it, D k-steps
// ahead in registers.  Their sums meet in LDS.  HBM bounds it: 1 row, us and TB/s of W: 4096 x 4096 4.9, 12288 x 4096 10.4 and 4.8, 22016 x 4096
// 16.6 and 5.4, 4096 x 11008 10.3 and 4.4 (4096 columns are one tile per CU: what is left there is the launch and a CU's first round trip).
template <int MT, int NT, int NW, int D, typename TO>
__global__ void __launch_bounds__(NW * 64) gemm_i8_kernel(I8Product p) {
  constexpr int kTiles = MT * NT;
  __shared__ i32x4 red[NW][kTiles][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = blockIdx.y * MT * 16, tile0 = blockIdx.x * NT;
  const int n_steps = p.K / kI8KStep;  // whole ones
  const int lo = (int)((int64_t)wave * n_steps / NW), hi = (int)((int64_t)(wave + 1) * n_steps / NW);
  const int8_t* xr[MT];
  const uint8_t* wr[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) xr[i] = p.X + (int64_t)min(row0 + i * 16 + (lane & 15), p.M - 1) * p.ldx + 16 * (lane >> 4);
#pragma unroll
  for (int j = 0; j < NT; ++j) wr[j] = p.W + (int64_t)min(tile0 + j, p.n_tiles - 1) * 16 * p.kp + lane * 16;
  i32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  i32x4 xb[D][MT], wb[D][NT];
  typedef i32x4 i32x4_any __attribute__((aligned(1)));
  auto load = [&](int b, int ks) {
    const int64_t k = min(ks, hi - 1);
#pragma unroll
    for (int j = 0; j < NT; ++j) wb[b][j] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(wr[j] + k * 1024));
#pragma unroll
    for (int i = 0; i < MT; ++i) xb[b][i] = *reinterpret_cast<const i32x4_any*>(xr[i] + k * kI8KStep);
  };
  auto multiply = [&](int b) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = mfma_i8(wb[b][j], xb[b][i], acc[i][j]);
  };
  if (lo < hi) {
#pragma unroll
    for (int b = 0; b < D; ++b) load(b, lo + b);
    int s = lo;
    for (; s + D <= hi; s += D)
#pragma unroll
      for (int b = 0; b < D; ++b) {
        multiply(b);
        load(b, s + b + D);
      }
#pragma unroll
    for (int b = 0; b < D; ++b)
      if (s + b < hi) multiply(b);
  }
  if (p.K % kI8KStep != 0 && wave == NW - 1) {  // the features behind the last whole k-step
#pragma unroll
    for (int j = 0; j < NT; ++j) wb[0][j] = *reinterpret_cast<const i32x4*>(wr[j] + (int64_t)n_steps * 1024);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int k = n_steps * kI8KStep + 16 * (lane >> 4);
      xb[0][i] = load_codes(xr[i] - 16 * (lane >> 4), k, p.K);
    }
    multiply(0);
  }
#pragma unroll
  for (int t = 0; t < kTiles; ++t) red[wave][t][lane] = acc[t / NT][t % NT];
  __syncthreads();
  for (int q = threadIdx.x; q < kTiles * 64; q += NW * 64) {
    const int t = q >> 6, l = q & 63;
    i32x4 sum = red[0][t][l];
#pragma unroll
    for (int w = 1; w < NW; ++w) sum += red[w][t][l];
    const int row = row0 + t / NT * 16 + (l & 15), tile = tile0 + t % NT, col = tile * 16 + 4 * (l >> 4);
    if (row < p.M && tile < p.n_tiles) store_scaled<TO>(p, row, col, sum, p.sx[row]);
  }
}

template <int MT, int NT, int NW, int D, typename TO>
static int launch_narrow(const I8Product& p, hipStream_t st) {
  MDZ_REQUIRE(i8_launchable((p.n_tiles + NT - 1) / NT, NW * 64), MDZ_EUNSUPPORTED, "linear_i8: %d columns are more than one launch takes", p.N);
  launch_timed(PROF_GEMM_I8, gemm_i8_kernel<MT, NT, NW, D, TO>, dim3((p.n_tiles + NT - 1) / NT, (p.M + MT * 16 - 1) / (MT * 16)), NW * 64, 0, st, p);
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

// Rows that do not start on 16 bytes, again 16 bytes apart and padded (with zeros) to whole k-steps.
__global__ void __launch_bounds__(256) align_rows_kernel(const int8_t* __restrict__ X, int K, i32x4* __restrict__ out, int64_t chunks, int per_row) {
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (q >= chunks) return;
  const int64_t row = q / per_row;
  out[q] = load_codes(X + row * K, (int)(q - row * per_row) * 16, K);
}

struct I8Plan {
  int tile;    // of kI8Tiles; -1: the kernel of few rows
  int splits;  // of the features
  int64_t aligned_at, bytes;  // workspace: the partial sums, then the rows aligned, where a call needs them
};

// Up to 16 rows take the kernel above; up to 32 do where neither the rows (K) nor the weights are long, because it loads a row in pieces of
// 64 bytes, a third slower than the tiles' 128 (us, this kernel / tiles: 24 rows 4096 x 4096 7.0 / 8.9, 32 rows 12288 x 4096 13.1 / 14.2;
// 22016 x 4096 22.8 / 21.1, 4096 x 11008 16.3 / 14.1).  Beyond, the tile and the number of splits of the least modelled time: the longest
// of what a CU needs for its workgroups, what the chip needs for all, and W from HBM, which idle CUs slow down; a split adds a launch and
// its sums' way to memory and back.  Fitted to 4500 timings (17 .. 2048 rows; 688 x 256, 864 x 7968 .. 22016 x 4096 and 5120 x 13824) of a build whose
// outputs left in another way; timed again with the present one, 228 products: what it picks takes 0.7 % longer than the best tile and split on
// average, 11 % at most (128 x 3696 x 4640).  The rule of up to 32 rows costs 2.9 % on average over 39 products, and up to 31 % where K is short and
// columns are many (32 x 14624 x 2096: 14.2 us, 10.9 in tiles).  All these K are multiples of 16: the copy of unaligned rows is in no cost.
// summed_later: the consumer adds the parts, so a split costs no launch, and has up to kI8MaxParts.  Nothing was fitted for it: timed with
// the norm that follows, 149 products, what it picks takes 1.4 % longer than the best on average, 19 % at most (384 x 5568 x 7008), and 10 % at 64 x 4096 x 4096
// (whole 12.7 us with the norm, in three parts 11.6).
static I8Plan plan_i8(int M, int N, int K, bool summed_later = false) {
  I8Plan best{-1, 1, 0, 0};
  if (M <= 16 || (M <= 32 && K <= 8192 && (int64_t)N * K <= 1 << 26)) return best;
  const int n_pad = (int)i8_padded_rows(N), stages = (K + 127) / 128, cus = num_cus();
  const float hbm = (float)N * K * (1e-6f / 7.0f);
  float least = 0.f;
  for (int t = 0; t < kNumI8Tiles; ++t) {
    const I8Tile& tile = kI8Tiles[t];
    if (t > 0 && tile.rows >= 2 * M) break;
    const int64_t blocks = (int64_t)((M + tile.rows - 1) / tile.rows) * ((N + tile.cols - 1) / tile.cols);
    for (int splits : {1, 2, 3, 4, 6, 8}) {
      if (splits > 1 && (splits * 4 > stages || blocks * splits > 4 * cus || (summed_later && splits > kI8MaxParts))) break;
      const int64_t wgs = blocks * splits;
      const float s = (float)((stages + splits - 1) / splits);
      const float rounds = (float)((wgs + cus - 1) / cus);
      const float cu = rounds * s * tile.us_stage * (rounds > 1.f && tile.two ? 0.81f : 1.f);
      float us = fmaxf(fmaxf(cu, (float)wgs * s * tile.us_all), hbm * sqrtf(rounds * cus / wgs)) + 0.33f * (rounds - 1.f);
      if (splits > 1) us += (summed_later ? 0.f : 1.6f) + (float)splits * M * n_pad * (4e-6f / 2.1f);
      if (best.tile < 0 || us < least) best.tile = t, best.splits = splits, least = us;
    }
  }
  best.aligned_at = best.splits > 1 ? best.splits * (int64_t)M * n_pad * 4 : 0;
  best.bytes = best.aligned_at + (int64_t)M * i8_padded_k(K);
  return best;
}

// One 16-column tile per workgroup until every CU has one, then two, then three, whose loads share the rows' (us at 1 row, one / two / three
// tiles: 4096 x 4096 4.9 / 5.9 / 7.0; 16 rows 6144 x 4096 9.1 / 7.3 / 8.4; 22016 x 4096 17.5 / 17.4 / 16.6)
static int few_rows_tiles(int n_tiles) { return n_tiles <= num_cus() ? 1 : n_tiles <= 2 * num_cus() ? 2 : 3; }
template <int MT, typename TO>
static int launch_few_rows(const I8Product& p, hipStream_t st) {
  switch (few_rows_tiles(p.n_tiles)) {
    case 1: return launch_narrow<MT, 1, 4, 4, TO>(p, st);
    case 2: return launch_narrow<MT, 2, 4, 4, TO>(p, st);
    default: return launch_narrow<MT, 3, 4, MT == 1 ? 6 : 4, TO>(p, st);
  }
}

static int check_linear_i8(int M, int N, int K) {
  MDZ_REQUIRE(M >= 0 && N > 0 && K > 0, MDZ_EINVAL, "linear_i8: [%d,%d] x [%d,%d]", M, K, N, K);
  MDZ_REQUIRE(K <= kI8MaxK, MDZ_EUNSUPPORTED, "linear_i8: up to %d input features, whose 32-bit sums cannot overflow (%d)", kI8MaxK, K);
  MDZ_REQUIRE(M <= 1 << 30 && N <= 1 << 30 && (int64_t)M * N < (int64_t)1 << 40, MDZ_EUNSUPPORTED, "linear_i8: %d x %d outputs", M, N);
  return MDZ_OK;
}

static I8Product describe(const int8_t* codes, const float* scales, const void* packed, int M, int N, int K, void* y) {
  I8Product p{};
  p.X = codes, p.sx = scales, p.W = (const uint8_t*)packed, p.sw = (const float*)((const char*)packed + i8_scales_offset(N, K)), p.Y = y;
  p.M = M, p.N = N, p.K = K, p.ldx = K, p.kp = i8_padded_k(K), p.n_tiles = (int)(i8_padded_rows(N) / kI8TileRows);
  return p;
}

// The tiles' loads take 16 bytes from addresses of 16: rows that do not start there go through the workspace.  Both launches' sizes are asked here,
// before the first of them.  (The parts of a split and the launch that adds them are few: plan_i8 splits up to 4 workgroups per CU.)
static int align_rows(I8Product& p, const I8Plan& plan, void* ws, hipStream_t st) {
  const bool aligned_already = p.K % 16 == 0 && reinterpret_cast<uintptr_t>(p.X) % 16 == 0;
  const int64_t chunks = (int64_t)p.M * (p.kp / 16);
  MDZ_REQUIRE(i8_launchable(i8_tile_workgroups(kI8Tiles[plan.tile], p.M, p.n_tiles), kI8Tiles[plan.tile].threads), MDZ_EUNSUPPORTED,
              "linear_i8: %d x %d outputs are more than one launch takes", p.M, p.N);
  MDZ_REQUIRE(aligned_already || i8_launchable((chunks + 255) / 256, 256), MDZ_EUNSUPPORTED,
              "linear_i8: %d unaligned rows are more than one launch takes", p.M);
  if (aligned_already) return MDZ_OK;
  i32x4* aligned = (i32x4*)((char*)ws + plan.aligned_at);
  launch_timed(PROF_GEMM_I8, align_rows_kernel, (unsigned)((chunks + 255) / 256), 256, 0, st, p.X, p.K, aligned, chunks, (int)(p.kp / 16));
  MDZ_LAUNCH_CHECK();
  p.X = (const int8_t*)aligned, p.ldx = p.kp, p.K = (int)p.kp;
  return MDZ_OK;
}

int64_t linear_i8_parts_bytes(int M, int N, int K) { return plan_i8(M, N, K, true).bytes; }

int launch_linear_i8_parts(const int8_t* codes, const float* scales, const void* packed, int M, int N, int K, float* y, void* ws, int64_t ws_bytes,
                           I8Sums* sums, hipStream_t st) {
  *sums = I8Sums{};
  const I8Plan plan = plan_i8(M, N, K, true);
  if (plan.splits == 1) return medusa_linear_i8(codes, scales, packed, M, N, K, MDZ_FP32, y, ws, ws_bytes, st);
  MDZ_REQUIRE(ws_bytes >= plan.bytes, MDZ_EWORKSPACE, "linear_i8: workspace %lld < %lld bytes", (long long)ws_bytes, (long long)plan.bytes);
  I8Product p = describe(codes, scales, packed, M, N, K, y);
  int rc = align_rows(p, plan, ws, st);
  if (rc || (rc = launch_i8_tile_parts(p, plan.tile, plan.splits, ws, st))) return rc;
  *sums = I8Sums{(const int32_t*)ws, plan.splits, p.n_tiles * 16, (int64_t)M * p.n_tiles * 16, scales, p.sw};
  return MDZ_OK;
}

}  // namespace mdz

using namespace mdz;

extern "C" {
#pragma GCC visibility push(default)

int64_t medusa_linear_i8_workspace_bytes(int M, int N, int K) {
  const int rc = check_linear_i8(M, N, K);
  return rc ? rc : plan_i8(M, N, K).bytes;
}

int medusa_linear_i8_plan(int M, int N, int K, int32_t* tile_rows, int32_t* tile_cols, int32_t* k_splits) {
  const int rc = check_linear_i8(M, N, K);
  if (rc) return rc;
  const I8Plan p = plan_i8(M, N, K);
  if (tile_rows) *tile_rows = p.tile >= 0 ? kI8Tiles[p.tile].rows : M <= 16 ? 16 : 32;
  if (tile_cols) *tile_cols = p.tile >= 0 ? kI8Tiles[p.tile].cols : 16 * few_rows_tiles((int)(i8_padded_rows(N) / kI8TileRows));
  if (k_splits) *k_splits = p.splits;
  return MDZ_OK;
}

int64_t medusa_linear_i8_parts_plan(int M, int N, int K, int32_t* k_splits) {
  const int rc = check_linear_i8(M, N, K);
  if (rc) return rc;
  if (k_splits) *k_splits = plan_i8(M, N, K, true).splits;
  const int64_t whole = plan_i8(M, N, K).bytes, parts = linear_i8_parts_bytes(M, N, K);
  return whole > parts ? whole : parts;
}

int medusa_test_i8_update_norm(int dtype, const int8_t* codes, const float* scales, const void* packed, int M, int d, int K, float* x,
                               const void* gain, float eps, int8_t* codes_out, float* scales_out, float* part, void* ws, int64_t ws_bytes,
                               void* stream) {
  MDZ_REQUIRE(is_16bit(dtype) && M > 0 && d > 0 && d % 32 == 0 && d <= kI8MaxPartsWidth, MDZ_EINVAL, "i8 update norm: dtype %d, [%d,%d]", dtype, M, d);
  MDZ_REQUIRE(codes && scales && packed && x && gain && codes_out && scales_out && part && reinterpret_cast<uintptr_t>(ws) % 16 == 0, MDZ_EINVAL,
              "i8 update norm: bad pointer");
  const int64_t need = medusa_linear_i8_parts_plan(M, d, K, nullptr);
  if (need < 0) return (int)need;
  MDZ_REQUIRE(ws_bytes >= need && (ws || need == 0), MDZ_EWORKSPACE, "i8 update norm: workspace %lld < %lld bytes", (long long)ws_bytes, (long long)need);
  I8Sums sums{};
  const int rc = launch_linear_i8_parts(codes, scales, packed, M, d, K, part, ws, ws_bytes, &sums, (hipStream_t)stream);
  if (rc) return rc;
  return launch_residual_rmsnorm_i8(dtype, x, part, sums, gain, eps, M, d, codes_out, scales_out, (hipStream_t)stream);
}

int medusa_linear_i8(const int8_t* codes, const float* scales, const void* packed, int M, int N, int K, int out_dtype, void* y, void* ws,
                     int64_t ws_bytes, void* stream) {
  MDZ_REQUIRE(dtype_ok(out_dtype), MDZ_EINVAL, "linear_i8: bad dtype %d", out_dtype);
  int rc = check_linear_i8(M, N, K);
  if (rc) return rc;
  if (M == 0) return MDZ_OK;
  MDZ_REQUIRE(codes && scales && packed && y, MDZ_EINVAL, "linear_i8: NULL pointer");
  MDZ_REQUIRE((reinterpret_cast<uintptr_t>(packed) & 15) == 0, MDZ_EINVAL, "linear_i8: the packed matrix must start on 16 bytes");
  MDZ_REQUIRE(reinterpret_cast<uintptr_t>(scales) % 4 == 0 && reinterpret_cast<uintptr_t>(y) % elem_bytes(out_dtype) == 0, MDZ_EINVAL,
              "linear_i8: a buffer is not aligned to its elements");
  const I8Plan plan = plan_i8(M, N, K);
  MDZ_REQUIRE(ws_bytes >= plan.bytes && (ws || plan.bytes == 0), MDZ_EWORKSPACE, "linear_i8: workspace %lld < %lld bytes",
              (long long)ws_bytes, (long long)plan.bytes);
  MDZ_REQUIRE(plan.bytes == 0 || (reinterpret_cast<uintptr_t>(ws) & 15) == 0, MDZ_EINVAL, "linear_i8: the workspace must start on 16 bytes");
  hipStream_t st = (hipStream_t)stream;
  I8Product p = describe(codes, scales, packed, M, N, K, y);
  if (plan.tile < 0) MDZ_WITH_ELEM(out_dtype, return (M <= 16 ? launch_few_rows<1, E>(p, st) : launch_few_rows<2, E>(p, st)));
  if ((rc = align_rows(p, plan, ws, st))) return rc;
  return launch_i8_tile(out_dtype, p, plan.tile, plan.splits, ws, st);
}

#pragma GCC visibility pop
}  // extern "C"
