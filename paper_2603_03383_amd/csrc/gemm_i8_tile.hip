// Product of 8-bit rows with packed 8-bit weights over more than 16 rows (32: see plan_i8): y = (sx sw^T) o (X W^T), sums in 32-bit integers,
// which are exact, so neither the tile, nor a split of the features, nor the number of rows changes a result.
//   * A workgroup owns a tile of the output.  X and W go straight to an LDS ring (`global_load_lds`, 16 bytes per lane, no registers) in
//     stages of 128 features: a cache line of each row of X, two k-steps of each tile of W.  One counted wait and one barrier per stage
//     make a stage everyone's; the stage that all have read is requested anew right behind it.
//   * The operands of a k-step (v_mfma_i32_16x16x64_i8) are read from LDS while the one before multiplies, across the barrier too (when it
//     was built in, 1024 x 22016 x 4096 gained 3 %, with 256 x 128 tiles 7 %).  The MFMA is issued as W x X^T: a lane ends with four columns of one row.
//   * X is row-major; its 16-byte chunks change places by the row's number on the way in, so that the reads take two clocks of the banks per
//     wave and 256 bytes, which is what they need (no conflicts are counted).  Read to registers in operand order instead, 16 rows x
//     64 bytes per load, X took three times as long as W's whole kilobytes (64 rows of 4096 x 4096: 13.1 us, 9.5 so; 12288: 17.7, 14.5).
// What bounds it.  Up to 64 rows how W is asked for, not the bytes that a CU can take in: 64 x 12288 x 4096 takes 14.9 us, 15.2 without the MFMAs and 13.7
// with W alone, which is 197 KB per CU; the kernel of few rows streams the same matrix in 9-10 us over as many workgroups, with up to 72 KB of W
// in flight per CU over four waves that wait for nobody, where here it is 30 KB behind a barrier per stage.  (Deeper rings changed nothing, so it
// is not the bytes in flight alone.)  From there to ~300 rows the bytes that the CUs take in, X once per column block and W once per row block:
// 11 to 19 TB/s over the chip, the smaller tiles more.  Hence tiles that go by the number of rows, and a split of the features where columns are
// few: parts of 64 x 64 tiles instead of whole sums of 64 x 16 (64 x 4096 x 11008: 20.6 us whole, 15.4 in four parts with the launch that
// adds them).  64 x 22016 x 4096: 18.5-21 us as W lies in the memory-side cache or not, 4.3-5 TB/s, against 19.0 at the rate of a large copy.
// With many rows: 256 x 192 tiles of eight waves, whose loads alone take 50 us per 256 tiles of 4096 features, the LDS reads and MFMAs 47,
// together 55-62; the matrix cores are 40 % busy and the clock falls with the codes' bits (zeros: 52).  1024 x 22016 x 4096: 100-117 us, 1.6-1.8
// Pop/s (a library product of the same shape without scales: 133); 1024 x 12288 x 4096: 55 (73); 1024 x 4096 x 11008: 56 (57).
// Tried and left out: stages of 64 features in deeper rings (half of each cache line of X per load: 5-20 % slower), W non-temporal (+-5 %
// either way), 256 x 256 tiles (344 of them on 256 CUs: 131 us), one wave per SIMD (155 us), a wave priority around the MFMAs (nothing).
#include "gemm_i8.h"
#include "gemm_rows.h"

namespace mdz {

// all but the youngest `n` stages of L loads each have landed, for n <= NS
template <int L, int NS>
__device__ inline void wait_stages(int n) {
  if (n >= NS) wait_loads<NS * L>();
  else static_for<NS>([&](auto i) {
    if (n == decltype(i)::value) wait_loads<decltype(i)::value * L>();
  });
}

constexpr int kI8Stage = 128;  // features of a stage of the ring: one cache line of a row of X, two k-steps of a tile of W

// Waves: WR x WC, each with MT 16-row tiles x NT 16-column tiles.  NS stages of the ring.  PARTIAL: a workgroup sums a part of the
// features (blockIdx.z) and writes its 32-bit sums to P[blockIdx.z], [M][n_tiles * 16].
template <int WR, int WC, int MT, int NT, int NS, typename TO, bool PARTIAL>
__global__ void __launch_bounds__(WR * WC * 64) gemm_i8_tile_kernel(I8Product p, i32x4* __restrict__ P, int nb_m, int nb_n, int splits) {
  constexpr int NW = WR * WC, XT = WR * MT, WT = WC * NT;  // waves; 16-row and 16-column tiles of the workgroup
  constexpr int UX = XT * 2, U = (XT + WT) * 2;            // 1 KiB pieces of a stage: X (8 rows x 128 features), then W (a k-step of a tile)
  constexpr int L = (U + NW - 1) / NW;                     // loads per wave and stage (a wave without a piece repeats the last)
  constexpr uint32_t kSlot = U * 1024;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds_raw[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / WC, wc = wave % WC;
  // Workgroups go round-robin to the 8 XCDs.  Each takes an eighth of the blocks, a column block's row blocks one after the other, so that they
  // share its weights through the XCD's L2.  (Whole column blocks to each XCD left three of them with 39 workgroups on 32 CUs at 1548 x 2432 x
  // 1024: 18.5 us, 11.0 so.)
  const int xcd = blockIdx.x & 7, blocks = nb_m * nb_n;
  const int block = (int)((int64_t)blocks * xcd >> 3) + (int)(blockIdx.x >> 3);
  if (block >= (int)((int64_t)blocks * (xcd + 1) >> 3)) return;
  const int bn = block / nb_m, bm = block % nb_m;
  const int n_stages = (p.K + kI8Stage - 1) / kI8Stage;
  const int lo = (int)((int64_t)blockIdx.z * n_stages / splits), n = (int)((int64_t)(blockIdx.z + 1) * n_stages / splits) - lo;
  const int row0 = bm * XT * 16, tile0 = bn * WT;
  const int last_row = p.M - 1 - row0, last_tile = p.n_tiles - 1 - tile0;
  const uint32_t lds0 = MDZ_LDS_ADDR(lds_raw);
  const uint8_t* x0 = reinterpret_cast<const uint8_t*>(p.X) + (int64_t)row0 * p.ldx + (int64_t)lo * kI8Stage;
  const uint8_t* w0 = p.W + (int64_t)tile0 * 16 * p.kp + (int64_t)lo * 2048;
  const uint32_t ldx = (uint32_t)p.ldx, tile_bytes = (uint32_t)p.kp * 16;
  // A piece of X: row lane / 8 of its eight, and the 16-byte chunk lane % 8, which changes places by the row's number so that the reads
  // spread over the banks.  Rows beyond M repeat the last and tiles beyond the matrix its last; neither is stored.
  const int chunk = ((lane & 7) ^ (lane >> 3)) * 16;
  auto load = [&](int s, int slot) {
    const uint32_t dst = lds0 + slot * kSlot;
    // (the last chunk again for those beyond K, whose weights are zero)
    const int at = min(chunk, p.K - 16 - (lo + s) * kI8Stage);
    static_for<L>([&](auto i) {
      constexpr int q = decltype(i)::value, first = q * NW, last = first + NW - 1;
      const int u = last < U ? first + wave : min(first + wave, U - 1);
      const uint8_t* const xp = x0 + (int64_t)s * kI8Stage;
      const uint8_t* const wp = w0 + (int64_t)s * 2048;
      const uint32_t xo = __umul24(min(u * 8 + (lane >> 3), last_row), ldx) + at;
      const uint32_t wo = (uint32_t)min((u - UX) >> 1, last_tile) * tile_bytes + ((u & 1) * 1024 + lane * 16);
      const bool of_x = last < UX || (first < UX && u < UX);
      load_to_lds<0>(of_x ? xp : wp, of_x ? xo : wo, dst + u * 1024);
    });
  };
  auto read = [&](i32x4(&a)[NT], i32x4(&b)[MT], int slot, int ks) {
    const uint8_t* xs = lds_raw + slot * kSlot;
    const uint8_t* ws = xs + UX * 1024;
    const int r = lane & 15, c = (ks * 4 + (lane >> 4)) ^ (r & 7);
#pragma unroll
    for (int j = 0; j < NT; ++j) a[j] = *reinterpret_cast<const i32x4*>(ws + ((wc * NT + j) * 2 + ks) * 1024 + lane * 16);
#pragma unroll
    for (int i = 0; i < MT; ++i) b[i] = *reinterpret_cast<const i32x4*>(xs + (wr * MT + i) * 2048 + r * 128 + c * 16);
  };

  i32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  auto multiply = [&](const i32x4(&a)[NT], const i32x4(&b)[MT]) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = mfma_i8(a[j], b[i], acc[i][j]);
  };

  static_for<NS>([&](auto i) {
    if (decltype(i)::value < n) load(decltype(i)::value, decltype(i)::value);
  });
  if (n > 0) {
    i32x4 a0[NT], b0[MT], a1[NT], b1[MT];  // the operands of a k-step are read while the one before multiplies
    wait_stages<L, NS - 1>(n - 1);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read(a0, b0, 0, 0);
    int slot = 0;
    for (int s = 0; s < n; ++s) {
      read(a1, b1, slot, 1);
      multiply(a0, b0);
      const int next = slot + 1 == NS ? 0 : slot + 1;
      if (s + 1 < n) {
        wait_lds();
        wait_stages<L, NS - 2>(n - 2 - s);  // this wave's loads of the next stage have landed, its reads of this one too
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + NS < n) load(s + NS, slot);
        read(a0, b0, next, 0);
      }
      multiply(a1, b1);
      slot = next;
    }
  }

#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int row = row0 + (wr * MT + i) * 16 + (lane & 15);
    if (row >= p.M) continue;
    const float sx = PARTIAL ? 0.f : p.sx[row];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int tile = tile0 + wc * NT + j, col = tile * 16 + 4 * (lane >> 4);
      if (tile >= p.n_tiles) continue;
      if constexpr (PARTIAL)
        P[(((int64_t)blockIdx.z * p.M + row) * p.n_tiles * 16 + col) >> 2] = acc[i][j];
      else
        store_scaled<TO>(p, row, col, acc[i][j], sx);
    }
  }
}

// y = scaled sum of the partial sums: a thread has four columns of a row
template <typename TO>
__global__ void __launch_bounds__(256) gemm_i8_finish_kernel(I8Product p, const i32x4* __restrict__ P, int splits) {
  const int64_t quads = (int64_t)p.M * p.n_tiles * 4, q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (q >= quads) return;
  i32x4 s = P[q];
  for (int z = 1; z < splits; ++z) s += P[z * quads + q];
  const int row = (int)(q / (p.n_tiles * 4)), col = (int)(q % (p.n_tiles * 4)) * 4;
  store_scaled<TO>(p, row, col, s, p.sx[row]);
}

template <int WR, int WC, int MT, int NT, int NS, typename TO, bool PARTIAL>
static int launch_tile(const I8Product& p, int splits, i32x4* partial, hipStream_t st) {
  constexpr int kLds = (WR * MT + WC * NT) * 2048 * NS;
  const int nb_m = (p.M + WR * MT * 16 - 1) / (WR * MT * 16), nb_n = (p.n_tiles + WC * NT - 1) / (WC * NT);
  auto kernel = gemm_i8_tile_kernel<WR, WC, MT, NT, NS, TO, PARTIAL>;
  MDZ_SET_LDS_ONCE(kernel, kLds);
  launch_timed(PROF_GEMM_I8, kernel, dim3((unsigned)(((int64_t)nb_m * nb_n + 7) / 8 * 8), 1, splits), WR * WC * 64, kLds, st, p, partial, nb_m, nb_n, splits);
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

// Waves (rows x columns of them), 16-row and 16-column tiles of a wave, stages of the ring, and the two times of I8Tile.  Few rows take wide
// rings of small stages (a CU's intake is the bound, and two workgroups per CU cover each other's start and end); many rows take the
// largest tiles, which need the fewest bytes per product.
#define MDZ_I8_TILES(T)          \
  T(2, 2, 1, 1, 8, .137, .421)   \
  T(4, 1, 1, 3, 5, .265, 1.02)   \
  T(2, 2, 2, 2, 4, .313, .945)   \
  T(4, 3, 1, 2, 4, .331, 1.61)   \
  T(2, 4, 3, 1, 5, .385, 1.49)   \
  T(2, 4, 4, 1, 4, .426, 1.80)   \
  T(2, 4, 4, 2, 4, .545, 2.63)   \
  T(4, 4, 4, 2, 3, .963, 3.82)   \
  T(4, 2, 4, 6, 2, 1.305, 5.16)
#define MDZ_I8_TILE_FACTS(WR, WC, MT, NT, NS, STAGE, ALL) \
  {WR * MT * 16, WC * NT * 16, WR * WC * 64, (WR * MT + WC * NT) * 2048 * NS <= 80 * 1024, STAGE##f, ALL##f * 1e-3f},
const I8Tile kI8Tiles[kNumI8Tiles] = {MDZ_I8_TILES(MDZ_I8_TILE_FACTS)};

template <typename TO, bool PARTIAL>
static int launch_by_tile(const I8Product& p, int tile, int splits, i32x4* partial, hipStream_t st) {
  int i = 0;
#define MDZ_I8_TILE_LAUNCH(WR, WC, MT, NT, NS, STAGE, ALL) \
  if (tile == i++) return launch_tile<WR, WC, MT, NT, NS, TO, PARTIAL>(p, splits, partial, st);
  MDZ_I8_TILES(MDZ_I8_TILE_LAUNCH)
  MDZ_FAIL(MDZ_EINVAL, "linear_i8: no tile %d", tile);
}

int launch_i8_tile_parts(const I8Product& p, int tile, int splits, void* partial, hipStream_t st) {
  return launch_by_tile<float, true>(p, tile, splits, (i32x4*)partial, st);
}

int launch_i8_tile(int out_dtype, const I8Product& p, int tile, int splits, void* partial, hipStream_t st) {
  if (splits == 1) MDZ_WITH_ELEM(out_dtype, return (launch_by_tile<E, false>(p, tile, 1, nullptr, st)));
  const int rc = launch_i8_tile_parts(p, tile, splits, partial, st);
  if (rc) return rc;
  const int64_t quads = (int64_t)p.M * p.n_tiles * 4;
  MDZ_WITH_ELEM(out_dtype, (launch_timed(PROF_GEMM_I8, gemm_i8_finish_kernel<E>, (unsigned)((quads + 255) / 256), 256, 0, st, p,
                                         (const i32x4*)partial, splits)));
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

}  // namespace mdz
