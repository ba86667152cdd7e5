// The kernel of the products with 4-bit weights; gemm_i4_*.hip hold its instances by storage type and groups per block of features.
#pragma once
#include "gemm_rows.h"
#include "i4.h"

namespace mdz {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

// Codes to 16-bit operands.  A field of four bits under a fixed exponent is a number with the code in its mantissa: 16 + q in bf16, 128 + q in
// binary16, both exact.  binary16 has a packed addition, which takes 128 + z off and leaves q - z, exact too.  bf16 has none: its products are
// made with 16 + q and the sum of x over the group, times 16 + z, is taken off them in fp32 (kOffset below): the sums are some six times
// larger than with q - z and lose that much in their last bits, 2^-24 relative to them.
template <typename E>
struct I4Elem;
template <>
struct I4Elem<bf16_t> {
  static constexpr uint32_t kMagic = 0x41804180u;
  static constexpr float kOffset = 16.f;  // left on each code
  static constexpr bool kSums = true;     // the products need the sums of x
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  __device__ static inline f32x4_t mfma(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  __device__ static inline uint32_t minus(uint32_t w, uint32_t) { return w; }
  __device__ static inline uint32_t zero_pair(int) { return 0; }
};
template <>
struct I4Elem<f16_t> {
  static constexpr uint32_t kMagic = 0x58005800u;
  static constexpr float kOffset = 0.f;
  static constexpr bool kSums = false;
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  __device__ static inline f32x4_t mfma(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  __device__ static inline uint32_t minus(uint32_t w, uint32_t zp) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, w) - __builtin_bit_cast(h2, zp));
  }
  __device__ static inline uint32_t zero_pair(int z) { return (0x5800u | (uint32_t)z << 3) * 0x00010001u; }  // 128 + z twice
};

template <typename E>
__device__ inline u32x4_t dequantise(uint32_t w, uint32_t zp) {
  constexpr uint32_t kMask = 0x00780078u, kMagic = I4Elem<E>::kMagic;
  const uint32_t r[4] = {(w & kMask) | kMagic, (w >> 4 & kMask) | kMagic, (w >> 8 & kMask) | kMagic,
                         (__builtin_amdgcn_alignbit(w, w, 12) & kMask) | kMagic};
  return u32x4_t{I4Elem<E>::minus(r[0], zp), I4Elem<E>::minus(r[1], zp), I4Elem<E>::minus(r[2], zp), I4Elem<E>::minus(r[3], zp)};
}

template <typename E>
__device__ inline float half_to_float(uint32_t word, int hi) { return hi ? Elem16<E>::hi(word) : Elem16<E>::lo(word); }

// four consecutive columns of a row, as one store wherever the row starts
template <typename T>
__device__ inline void store_four(T* y, int left, f32x4_t v) {
  struct Four {
    T v[4];
  };
  typedef uint32_t Bits __attribute__((ext_vector_type(sizeof(Four) / 4)));
  typedef Bits Any __attribute__((aligned(1)));
  const Four f{{from_float<T>(v.x), from_float<T>(v.y), from_float<T>(v.z), from_float<T>(v.w)}};
  if (left >= 4) {
    *reinterpret_cast<Any*>(y) = __builtin_bit_cast(Bits, f);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) y[e] = f.v[e];
  }
}

// A workgroup of NW waves makes 16 MT rows x NT tiles of 16 columns (GATED: NT / 2 of each matrix); the waves share out the blocks of
// features, so each streams contiguous weights, and their sums meet in LDS.  A wave's rows of X pass through LDS of its own, which turns whole
// lines of memory into operands; no wave waits for another before the end.  XR: pieces of four rows that are loaded (4 MT, or fewer).
template <typename E, int G, bool ZEROS, bool GATED, int MT, int NT, int XR, int NW, int D>
__global__ void __launch_bounds__(NW * 64) gemm_i4_kernel(I4Product p) {
  typedef I4Elem<E> El;
  constexpr int kTiles = MT * NT, kGateTiles = GATED ? NT / 2 : NT;
  constexpr int kSteps = 4 / G;  // MFMA steps of a group
  typedef u32x4_t Any16 __attribute__((aligned(1)));
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds_raw[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q4 = lane >> 4, r16 = lane & 15;
  // Workgroups go round-robin to the 8 XCDs: each takes an eighth of the blocks, a column block's row blocks one after the other.
  const int xcd = blockIdx.x & 7, blocks = p.nb_m * p.nb_n;
  const int block = (int)((int64_t)blocks * xcd >> 3) + (int)(blockIdx.x >> 3);
  if (block >= (int)((int64_t)blocks * (xcd + 1) >> 3)) return;
  const int row0 = block % p.nb_m * MT * 16, tile0 = block / p.nb_m * kGateTiles;
  const int lo = (int)((int64_t)wave * p.n_blocks / NW), hi = (int)((int64_t)(wave + 1) * p.n_blocks / NW);
  const int last_row = p.M - 1 - row0;

  const uint16_t* const x0 = reinterpret_cast<const uint16_t*>(p.X) + (int64_t)row0 * p.K;
  const uint8_t* cp[NT];
  const uint8_t* sp[NT];
  const uint8_t* zp[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const I4Matrix& w = p.w[j >= kGateTiles];
    const int64_t at = (int64_t)min(tile0 + j % kGateTiles, p.n_tiles - 1) * p.n_blocks;
    cp[j] = w.codes + at * 1024 + lane * 16;
    sp[j] = w.scales + at * (32 * G) + q4 * (8 * G);
    zp[j] = ZEROS ? w.zeros + at * (16 * G) + (El::kSums ? q4 * (4 * G) : r16 * G) : nullptr;
  }
  // what a wave has requested of a block: X in pieces of 4 rows x 256 bytes, codes, scales, zero points
  constexpr int kScaleWords = 2 * G, kZeroWords = El::kSums ? G : 1;
  struct Scales {
    uint32_t w[kScaleWords];
  };
  struct Zeros {
    uint32_t w[kZeroWords];
  };
  u32x4_t xb[XR], cb[D][NT];
  Scales sb[D][NT];
  Zeros zb[D][NT];
  auto load_x = [&](int b) {
    const int k = min(b, hi - 1) * kI4Block + r16 * 8;
#pragma unroll
    for (int i = 0; i < XR; ++i) {
      const uint16_t* row = x0 + (int64_t)min(i * 4 + q4, last_row) * p.K;
      if (k + 8 <= p.K) {
        xb[i] = *reinterpret_cast<const Any16*>(row + k);
      } else {  // the features behind the last: zeros
        uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (k + e < p.K) v[e >> 1] |= (uint32_t)row[k + e] << 16 * (e & 1);
        xb[i] = u32x4_t{v[0], v[1], v[2], v[3]};
      }
    }
  };
  auto load_w = [&](int slot, int b) {
    const int64_t at = min(b, hi - 1);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      cb[slot][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(cp[j] + at * 1024));
      sb[slot][j] = *reinterpret_cast<const Scales*>(sp[j] + at * (32 * G));
      if constexpr (ZEROS) {
        const uint8_t* z = zp[j] + at * (16 * G);
        if constexpr (El::kSums) zb[slot][j] = *reinterpret_cast<const Zeros*>(z);
        else zb[slot][j].w[0] = G == 1 ? *z : G == 2 ? *reinterpret_cast<const uint16_t*>(z) : *reinterpret_cast<const uint32_t*>(z);
      }
    }
  };
  uint8_t* const xs = lds_raw + wave * (XR * 1024);

  f32x4_t tot[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) tot[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto block_of_features = [&](int slot, int next_x) {
    // 16-byte chunk c of a row stands at place c ^ (row % 16) of its 256 bytes, so that 16 rows' chunks are read without bank conflicts
#pragma unroll
    for (int i = 0; i < XR; ++i) {
      const int row = i * 4 + q4;
      *reinterpret_cast<u32x4_t*>(xs + row * 256 + ((r16 ^ (row & 15)) * 16)) = xb[i];
    }
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
    load_x(next_x);
    u32x4_t x[4][MT];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int row = min(i * 16 + r16, XR * 4 - 1);
        x[s][i] = *reinterpret_cast<const u32x4_t*>(xs + row * 256 + (((s * 4 + q4) ^ (row & 15)) * 16));
      }
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
    float sums[G][MT];
    if constexpr (El::kSums) {
      const u32x4_t ones{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          f32x4_t a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < kSteps; ++s) a = El::mfma(ones, x[g * kSteps + s][i], a);
          sums[g][i] = a.x;
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        uint32_t zpair = El::zero_pair(8);
        if constexpr (ZEROS && !El::kSums) zpair = El::zero_pair(zb[slot][j].w[0] >> (8 * g) & 0xFFu);
        f32x4_t acc[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = g * kSteps; s < (g + 1) * kSteps; ++s) {
          const u32x4_t w = dequantise<E>(cb[slot][j][s], zpair);
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[i] = El::mfma(w, x[s][i], acc[i]);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int at = c * G + g;
          const float scale = half_to_float<E>(sb[slot][j].w[at >> 1], at & 1);
          float off = -(El::kOffset + 8.f);
          if constexpr (ZEROS && El::kSums) off = -El::kOffset - (float)(zb[slot][j].w[at >> 2] >> (8 * (at & 3)) & 0xFFu);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const float v = El::kSums ? fmaf(off, sums[g][i], acc[i][c]) : acc[i][c];
            tot[i][j][c] = fmaf(scale, v, tot[i][j][c]);
          }
        }
      }
    }
  };

  if (lo < hi) {
    load_x(lo);
#pragma unroll
    for (int d = 0; d < D; ++d) load_w(d, lo + d);
    int b = lo;
    for (; b + D <= hi; b += D)
#pragma unroll
      for (int d = 0; d < D; ++d) {
        block_of_features(d, b + d + 1);
        load_w(d, b + d + D);
      }
#pragma unroll
    for (int d = 0; d < D; ++d)
      if (b + d < hi) block_of_features(d, b + d + 1);
  }

  __syncthreads();
  f32x4_t* const red = reinterpret_cast<f32x4_t*>(lds_raw);  // [wave][tile][lane]
#pragma unroll
  for (int t = 0; t < kTiles; ++t) red[(wave * kTiles + t) * 64 + lane] = tot[t / NT][t % NT];
  __syncthreads();
  for (int t = wave; t < MT * kGateTiles; t += NW) {
    const int i = t / kGateTiles, j = t % kGateTiles;
    auto sum = [&](int tile) {
      f32x4_t v = red[tile * 64 + lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) v += red[(w * kTiles + tile) * 64 + lane];
      return v;
    };
    f32x4_t v = sum(i * NT + j);
    if constexpr (GATED) {
      const f32x4_t up = sum(i * NT + kGateTiles + j);
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = silu_tile(v[c]) * up[c];
    }
    const int row = row0 + i * 16 + r16, col = (tile0 + j) * 16 + 4 * q4;
    if (row >= p.M || col >= p.N) continue;
    const int64_t at = (int64_t)row * p.N + col;
    if (!GATED && p.out_dtype == MDZ_FP32) store_four(reinterpret_cast<float*>(p.Y) + at, p.N - col, v);
    else if (!GATED && p.out_dtype != (__is_same(E, bf16_t) ? MDZ_BF16 : MDZ_FP16))
      store_four(reinterpret_cast<std::conditional_t<__is_same(E, bf16_t), f16_t, bf16_t>*>(p.Y) + at, p.N - col, v);
    else store_four(reinterpret_cast<E*>(p.Y) + at, p.N - col, v);
  }
}

template <typename E, int G, bool ZEROS, bool GATED, int MT, int NT, int XR, int NW, int D>
static int launch_i4_kernel(I4Product p, hipStream_t st) {
  constexpr int kGateTiles = GATED ? NT / 2 : NT;
  constexpr int kLds = NW * 1024 * (XR > MT * NT ? XR : MT * NT);
  p.nb_m = (p.M + MT * 16 - 1) / (MT * 16), p.nb_n = (p.n_tiles + kGateTiles - 1) / kGateTiles;
  const int64_t workgroups = ((int64_t)p.nb_m * p.nb_n + 7) / 8 * 8;
  MDZ_REQUIRE(workgroups * NW * 64 <= (int64_t)UINT32_MAX, MDZ_EUNSUPPORTED, "linear_i4: %d x %d outputs are more than one launch takes", p.M, p.N);
  auto kernel = gemm_i4_kernel<E, G, ZEROS, GATED, MT, NT, XR, NW, D>;
  MDZ_SET_LDS_ONCE(kernel, kLds);
  launch_timed(PROF_GEMM_I4, kernel, dim3((unsigned)workgroups), NW * 64, kLds, st, p);
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

template <typename E, int G, bool ZEROS, bool GATED>
static int launch_i4_tiles(const I4Product& p, const I4Plan& plan, hipStream_t st) {
#define MDZ_I4_CASE(MT, NT, XR, NW, D) \
  if (plan.mt == MT && plan.nt == NT) return launch_i4_kernel<E, G, ZEROS, GATED, MT, NT, XR, NW, D>(p, st);
  MDZ_I4_CASE(1, 2, 4, 4, 4)
  MDZ_I4_CASE(4, 2, 16, 4, 2)
  MDZ_FAIL(MDZ_EINVAL, "linear_i4: no kernel of %d x %d tiles", plan.mt, plan.nt);
}

template <typename E, int G>
int launch_i4(const I4Product& p, bool zeros, bool gated, const I4Plan& plan, hipStream_t st) {
  if (zeros) return gated ? launch_i4_tiles<E, G, true, true>(p, plan, st) : launch_i4_tiles<E, G, true, false>(p, plan, st);
  return gated ? launch_i4_tiles<E, G, false, true>(p, plan, st) : launch_i4_tiles<E, G, false, false>(p, plan, st);
}

}  // namespace mdz
