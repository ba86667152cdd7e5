// The kernel of the products with 4-bit weights; gemm_i4_*.hip hold its instances by storage type and groups per block of features.
#pragma once
#include "gemm_rows.h"
#include "i4.h"

namespace mdz {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

// Codes to 16-bit operands.  A field of four bits at the top of a mantissa, under the exponent of 16, is 16 + q: one mask and one exponent make two
// operands of a word.  The products are made with 16 + q; what is too much, (16 + z) times the sum of x over the group, is taken off in fp32.  The sums
// are then some six times larger than with q - z and lose that much in their last bits, 2^-24 relative to them.  binary16 matrices with zero points in
// groups of 32 or 64 take (16 + q) - (16 + z) instead, which is exact: binary16 has a packed subtraction (bf16 has none), 16 instructions per tile and
// block in place of one FMA per output and group, and fewer registers (gated 200 x 12800 x 4096 in groups of 64: 94 -> 88 us, of 32: 210 -> 104; of 128
// it loses, 73 -> 77).
// The mask and the exponent are kept from the compiler as constants: from registers (w & mask) | magic is one instruction, from literals two.  (No
// inline assembly for it: the wait between a vector instruction and the MFMA that reads its result is the compiler's to see.)
constexpr float kI4Offset = 16.f;
template <typename E>
struct I4Elem;
template <>
struct I4Elem<bf16_t> {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  static constexpr uint32_t kMask = 0x00780078u, kMagic = 0x41804180u, kOne = 0x3F803F80u, kMinus24 = 0xC1C0C1C0u;
  __device__ static inline f32x4_t mfma(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};
template <>
struct I4Elem<f16_t> {
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  static constexpr uint32_t kMask = 0x03C003C0u, kMagic = 0x4C004C00u, kOne = 0x3C003C00u, kMinus24 = 0xCE00CE00u;
  __device__ static inline f32x4_t mfma(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};
template <typename E>
struct I4Constants {
  uint32_t mask = I4Elem<E>::kMask, magic = I4Elem<E>::kMagic;
  __device__ inline I4Constants() { asm volatile("" : "+s"(mask), "+v"(magic)); }
};
// features 2 i and 2 i + 1 of a word stand 4 i bits above the mask (i4_rotation)
template <typename E>
__device__ inline u32x4_t dequantise(uint32_t w, const I4Constants<E>& c) {
  return u32x4_t{(w & c.mask) | c.magic, (w >> 4 & c.mask) | c.magic, (__builtin_amdgcn_alignbit(w, w, 8) & c.mask) | c.magic,
                 (__builtin_amdgcn_alignbit(w, w, 12) & c.mask) | c.magic};
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

// of a block: scales of four rows, and their zero points; or (kI4Subtract) the zero points of the row that a lane's codes are of
template <int G>
struct I4Scales {
  uint32_t w[2 * G];
};
template <typename E, int G>
constexpr bool kI4Subtract = i4_subtracts(__is_same(E, f16_t), G);
template <typename E, int G>
struct I4Zeros {
  static constexpr int kStep = kI4Subtract<E, G> ? G : 4 * G;  // bytes from one to the next
  typedef std::conditional_t<G == 1, uint8_t, std::conditional_t<G == 2, uint16_t, uint32_t>> Row;
  uint32_t w[kI4Subtract<E, G> ? 1 : G];
  __device__ static inline int which(int lane) { return kI4Subtract<E, G> ? lane & 15 : lane >> 4; }
  __device__ inline void load(const uint8_t* at) {
    if constexpr (kI4Subtract<E, G>) w[0] = *reinterpret_cast<const Row*>(at);
    else *this = *reinterpret_cast<const I4Zeros*>(at);
  }
};
// uniform bases of a wave's tiles, and a lane's place in a block
template <typename E, int G, bool ZEROS, bool GATED, int NT>
struct I4Stream {
  static constexpr int kGateTiles = GATED ? NT / 2 : NT;
  const uint8_t* codes[NT];
  const uint8_t* scales[NT];
  const uint8_t* zeros[NT];
  uint32_t co, so, zo;
  __device__ inline I4Stream(const I4Product& p, int tile0, int lane) {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const I4Matrix& w = p.w[j >= kGateTiles];
      const int64_t at = (int64_t)min(tile0 + j % kGateTiles, p.n_tiles - 1) * p.n_blocks;
      codes[j] = w.codes + at * 1024;
      scales[j] = w.scales + at * (32 * G);
      zeros[j] = ZEROS ? w.zeros + at * (16 * G) : nullptr;
    }
    co = lane * 16, so = (lane >> 4) * (8 * G), zo = I4Zeros<E, G>::which(lane) * I4Zeros<E, G>::kStep;
  }
  __device__ inline void load(u32x4_t (&c)[NT], I4Scales<G> (&s)[NT], I4Zeros<E, G> (&z)[NT], int b) const {
    const int64_t at = __builtin_amdgcn_readfirstlane(b);
    // A block's address is uniform and a lane's place in it 32 bits (kept from the compiler, which would make 64-bit vector addresses of them).
    uint32_t c0 = co, s0 = so, z0 = zo;
    asm volatile("" : "+v"(c0), "+v"(s0), "+v"(z0));
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const u32x4_t* const cp = reinterpret_cast<const u32x4_t*>(codes[j] + at * 1024 + c0);
      c[j] = __builtin_nontemporal_load(cp);
      s[j] = *reinterpret_cast<const I4Scales<G>*>(scales[j] + at * (32 * G) + s0);
      if constexpr (ZEROS) z[j].load(zeros[j] + at * (16 * G) + z0);
    }
  }
};

// What the products with 16 + q have too much, by the matrix cores: -24 times the sums of x over the groups, which the sums of a matrix without zero
// points start from, or the sums themselves.  x[s][i]: the operands of a block's four steps.
template <typename E, int G, bool ZEROS, int MT>
__device__ inline void sum_block(f32x4_t (&c0)[G][MT], const u32x4_t (&x)[4][MT]) {
  if constexpr (ZEROS && kI4Subtract<E, G>) return;
  constexpr uint32_t kFactor = ZEROS ? I4Elem<E>::kOne : I4Elem<E>::kMinus24;
  const u32x4_t factor{kFactor, kFactor, kFactor, kFactor};
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      f32x4_t a{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = g * (4 / G); s < (g + 1) * (4 / G); ++s) a = I4Elem<E>::mfma(factor, x[s][i], a);
      c0[g][i] = a;
    }
}

// tot += the products of one block of features and one tile of columns
template <typename E, int G, bool ZEROS, int MT>
__device__ inline void multiply_tile(f32x4_t (&tot)[MT], const u32x4_t (&x)[4][MT], const f32x4_t (&c0)[G][MT], u32x4_t codes, const I4Scales<G>& scales,
                                     const I4Zeros<E, G>& zeros, const I4Constants<E>& constants) {
  constexpr int kSteps = 4 / G;  // MFMA steps of a group
  constexpr bool kSubtract = ZEROS && kI4Subtract<E, G>;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    f32x4_t acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = ZEROS ? f32x4_t{0.f, 0.f, 0.f, 0.f} : c0[g][i];
#pragma unroll
    for (int s = g * kSteps; s < (g + 1) * kSteps; ++s) {
      const uint32_t word = codes[s];
      u32x4_t w = dequantise<E>(word, constants);
      if constexpr (kSubtract) {
        typedef _Float16 Eight __attribute__((ext_vector_type(8)));
        const uint32_t z = 0x4C00u | (zeros.w[0] >> (8 * g) & 0xFFu) << 6;  // 16 + z
        const uint32_t two = z | z << 16;
        w = __builtin_bit_cast(u32x4_t, __builtin_bit_cast(Eight, w) - __builtin_bit_cast(Eight, u32x4_t{two, two, two, two}));
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) acc[i] = I4Elem<E>::mfma(w, x[s][i], acc[i]);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int at = c * G + g;
      const float scale = half_to_float<E>(scales.w[at >> 1], at & 1);
      constexpr bool kTakeOff = ZEROS && !kSubtract;
      const float off = kTakeOff ? -kI4Offset - (float)(zeros.w[kTakeOff ? at >> 2 : 0] >> (8 * (at & 3)) & 0xFFu) : 0.f;
#pragma unroll
      for (int i = 0; i < MT; ++i) tot[i][c] = fmaf(scale, kTakeOff ? fmaf(off, c0[g][i].x, acc[i][c]) : acc[i][c], tot[i][c]);
    }
  }
}

// Sums over WK waves that made the same outputs of their parts of the features (wk: which of them), the activation, and the way out.  `red`: LDS of WK x MT x NT KiB,
// not used where WK is 1.
template <typename E, bool GATED, int MT, int NT, int WK>
__device__ inline void finish_i4(const I4Product& p, const f32x4_t (&tot)[NT][MT], f32x4_t* red, int row0, int tile0, int wk, int lane) {
  constexpr int kTiles = MT * NT, kGateTiles = GATED ? NT / 2 : NT;
  auto put = [&](int i, int j, f32x4_t v, f32x4_t up) {
    if constexpr (GATED) {
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = silu_tile(v[c]) * up[c];
    }
    const int row = row0 + i * 16 + (lane & 15), col = (tile0 + j) * 16 + 4 * (lane >> 4);
    if (row >= p.M || col >= p.N) return;
    const int64_t at = (int64_t)row * p.N + col;
    if (!GATED && p.out_dtype == MDZ_FP32) store_four(reinterpret_cast<float*>(p.Y) + at, p.N - col, v);
    else if (!GATED && p.out_dtype != (__is_same(E, bf16_t) ? MDZ_BF16 : MDZ_FP16))
      store_four(reinterpret_cast<std::conditional_t<__is_same(E, bf16_t), f16_t, bf16_t>*>(p.Y) + at, p.N - col, v);
    else store_four(reinterpret_cast<E*>(p.Y) + at, p.N - col, v);
  };
  if constexpr (WK == 1) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < kGateTiles; ++j) put(i, j, tot[j][i], tot[GATED ? kGateTiles + j : j][i]);
  } else {
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTiles; ++t) red[(wk * kTiles + t) * 64 + lane] = tot[t % NT][t / NT];  // [part][tile][lane]
    __syncthreads();
    auto sum = [&](int tile) {
      f32x4_t v = red[tile * 64 + lane];
#pragma unroll
      for (int w = 1; w < WK; ++w) v += red[(w * kTiles + tile) * 64 + lane];
      return v;
    };
    for (int t = wk; t < MT * kGateTiles; t += WK) {
      const int i = t / kGateTiles, j = t % kGateTiles;
      put(i, j, sum(i * NT + j), GATED ? sum(i * NT + kGateTiles + j) : f32x4_t{});
    }
  }
}

// A workgroup of NW waves makes 16 MT rows x NT tiles of 16 columns (GATED: NT / 2 of each matrix); the waves share out the blocks of
// features, so each streams contiguous weights, and their sums meet in LDS.  A wave's rows of X pass through LDS of its own, which turns whole
// lines of memory into operands; no wave waits for another before the end.  XR: pieces of four rows that are loaded (4 MT, or fewer).
// Bound by the stream of weights at few rows: 1 x 12288 x 4096 in 8.5 us, 3.0 TB/s with the launch and the first loads in it, gated 1 x 11008 x 4096 12.9, 3.6 TB/s (registers
// hold 4 to 8 blocks per wave ahead; LDS would add a step that few rows do not need).  At 64 rows by loads, LDS, conversions and products one after the other, with all of X
// through every workgroup: 64 x 4096 x 4096 9.7 us, gated 64 x 11008 x 4096 24.1, where the ring below takes 31 and 32 (32 and 172 workgroups).  With one tile to a wave
// half of the products are those that make the sums of x.
template <typename E, int G, bool ZEROS, bool GATED, int MT, int NT, int XR, int NW, int D, int DX, int WPE>
__global__ void __launch_bounds__(NW * 64, WPE) gemm_i4_kernel(I4Product p) {
  typedef I4Stream<E, G, ZEROS, GATED, NT> Stream;
  typedef u32x4_t Any16 __attribute__((aligned(1)));
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds_raw[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q4 = lane >> 4, r16 = lane & 15;
  const int row0 = blockIdx.y * MT * 16, tile0 = blockIdx.x * Stream::kGateTiles;
  const int lo = (int)((int64_t)wave * p.n_blocks / NW), hi = (int)((int64_t)(wave + 1) * p.n_blocks / NW);
  const int last_row = p.M - 1 - row0;
  const uint8_t* const x0 = reinterpret_cast<const uint8_t*>(p.X) + (int64_t)row0 * p.K * 2;
  const Stream stream(p, tile0, lane);
  u32x4_t xb[DX][XR], cb[D][NT];
  I4Scales<G> sb[D][NT];
  I4Zeros<E, G> zb[D][NT];
  uint32_t xo[XR];
#pragma unroll
  for (int i = 0; i < XR; ++i) xo[i] = (uint32_t)min(i * 4 + q4, last_row) * (uint32_t)(2 * p.K) + r16 * 16;
  const int whole = p.K / kI4Block, end = min(hi, whole);  // whole blocks of features, and this wave's
  auto load_x = [&](int slot, int b) {
    const uint8_t* const at = x0 + (int64_t)__builtin_amdgcn_readfirstlane(min(b, end - 1)) * (2 * kI4Block);
#pragma unroll
    for (int i = 0; i < XR; ++i) {
      uint32_t o = xo[i];
      asm volatile("" : "+v"(o));
      xb[slot][i] = *reinterpret_cast<const Any16*>(at + o);
    }
  };
  uint8_t* const xs = lds_raw + wave * (XR * 1024);

  f32x4_t tot[NT][MT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) tot[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // the rows' block to LDS: 16-byte chunk c of a row stands at place c ^ (row % 16) of its 256 bytes, so that 16 rows' chunks are read without
  // bank conflicts
  auto put_x = [&](int slot) {
#pragma unroll
    for (int i = 0; i < XR; ++i) {
      const int row = i * 4 + q4;
      *reinterpret_cast<u32x4_t*>(xs + row * 256 + ((r16 ^ (row & 15)) * 16)) = xb[slot][i];
    }
  };
  // the features behind the last whole block, and zeros behind them: each lane loads the 16 bytes from its place on, or where the row ends before, those that
  // end with it, and moves them down (one load per piece and all under way together: one by one the features of 64 rows took 17 us)
  auto load_last_x = [&]() {
    const int k = whole * kI4Block + r16 * 8, at = min(k, p.K - 8);
#pragma unroll
    for (int i = 0; i < XR; ++i) {
      const uint8_t* const row = x0 + (uint32_t)min(i * 4 + q4, last_row) * (uint32_t)(2 * p.K);
      uint64_t lo = 0, hi = 0;
      if (at >= 0) {
        typedef uint64_t Two __attribute__((ext_vector_type(2)));
        typedef Two AnyTwo __attribute__((aligned(1)));
        const Two v = *reinterpret_cast<const AnyTwo*>(row + 2 * (int64_t)at);
        lo = v.x, hi = v.y;
        const int down = 16 * (k - at);  // bits
        if (down >= 64) lo = hi >> (down & 63), hi = 0;
        else if (down > 0) lo = lo >> down | hi << (64 - down), hi >>= down;
        if (down >= 128) lo = 0;
      } else {  // fewer than 8 features in all
        for (int e = 0; k + e < p.K; ++e) {
          const uint64_t one = reinterpret_cast<const uint16_t*>(row)[k + e];
          if (e < 4) lo |= one << (16 * e);
          else hi |= one << (16 * (e - 4));
        }
      }
      xb[0][i] = u32x4_t{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
    }
  };
  const I4Constants<E> constants;
  auto multiply = [&](int slot) {
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
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
    f32x4_t c0[G][MT];
    sum_block<E, G, ZEROS>(c0, x);
#pragma unroll
    for (int j = 0; j < NT; ++j) multiply_tile<E, G, ZEROS>(tot[j], x, c0, cb[slot][j], sb[slot][j], zb[slot][j], constants);
    // (pure arithmetic would be put off past the next blocks, with all that it needs kept in registers)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) asm volatile("" : "+v"(tot[j][i]));
  };

  if (hi > whole && lo < hi) {
    stream.load(cb[0], sb[0], zb[0], whole);
    load_last_x();
    put_x(0);
    multiply(0);
  }
  if (lo < end) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      if (d < DX) load_x(d, lo + d);
      stream.load(cb[d], sb[d], zb[d], min(lo + d, end - 1));
    }
    // (one way through the loop: the compiler's waits count requests, and take the least of all ways that lead to a place)
    for (int b = lo;; b += D)
#pragma unroll
      for (int d = 0; d < D; ++d) {
        put_x(d % DX);
        load_x(d % DX, b + d + DX);
        multiply(d);
        stream.load(cb[d], sb[d], zb[d], min(b + d + D, end - 1));
        if (b + d + 1 >= end) goto done;
      }
  }
done:

  finish_i4<E, GATED, MT, NT, NW>(p, tot, reinterpret_cast<f32x4_t*>(lds_raw), row0, tile0, wave, lane);
}

// More rows.  A workgroup makes 16 MT rows x NW NT tiles of columns with NW waves, which share the rows.  X, codes, scales and zero points go straight to an
// LDS ring of two turns (`global_load_lds`, 16 bytes per lane, no registers), a turn for each block of features; one wait and one barrier make a turn
// everyone's, and behind it the place of the turn that all have read is requested anew.  Two turns, so that a CU has two workgroups or three: their phases of
// loads, LDS reads, conversions and products then overlap.  (One workgroup of eight waves and three turns, all in step: gated 1024 x 11008 x 4096 219 us
// where two of four waves take 200, 64 x 128000 x 4096 85 and 81.)
// Bound by the matrix cores and the vector units, which convert codes and scale sums: gated 1024 x 11008 x 4096 in 189-195 us (0.95-0.98 PFLOP/s; each is busy for half of the
// clocks, and they overlap little), gated 200 x 12800 x 4096 in groups of 64 with zero points 86-88, 64 x 128000 x 4096 84-86 (3.6 TB/s).  A fifth of the matrix cores' clocks are
// the sums of x, which each wave makes for itself (sum_block).  64 rows to a wave, so that a converted tile serves four products; 256 columns to four waves, or
// 128 where that fills the CUs better (kI4Cuts).
template <int G, bool ZEROS, bool GATED, int MT, int NT, int NW>
struct I4Ring {
  static constexpr int kRows = MT * 16, kMats = GATED ? 2 : 1, kTiles = NW * NT / kMats;  // tiles of each matrix
  // 1 KiB pieces of a block: X (four rows), codes (a tile), scales, zero points
  static constexpr int kX = kRows / 4, kScales = (kTiles * 32 * G + 1023) / 1024, kZeros = ZEROS ? (kTiles * 16 * G + 1023) / 1024 : 0;
  static constexpr int kAtScales = kX + kMats * kTiles, kAtZeros = kAtScales + kMats * kScales, kPieces = kAtZeros + kMats * kZeros;
  static constexpr int kLoads = (kPieces + NW - 1) / NW;  // per turn and wave
  static constexpr int kTurn = kPieces * 1024, kLds = 2 * kTurn;
};
// a pointer that is the same in every lane, in scalar registers
__device__ inline const uint8_t* uniform(const uint8_t* p) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  // (the builtin gives a signed int)
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(a >> 32)), lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)a);
  return reinterpret_cast<const uint8_t*>((uint64_t)hi << 32 | lo);
}
template <typename E, int G, bool ZEROS, bool GATED, int MT, int NT, int NW, int WPE>
__global__ void __launch_bounds__(NW * 64, WPE) gemm_i4_rows_kernel(I4Product p) {
  typedef I4Ring<G, ZEROS, GATED, MT, NT, NW> R;
  constexpr int L = R::kLoads;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds_raw[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q4 = lane >> 4, r16 = lane & 15;
  // Workgroups go round-robin to the 8 XCDs: each takes an eighth of the blocks, a column block's row blocks one after the other, which then
  // share its weights through the XCD's L2.
  const int xcd = blockIdx.x & 7, blocks = p.nb_m * p.nb_n;
  const int block = (int)((int64_t)blocks * xcd >> 3) + (int)(blockIdx.x >> 3);
  if (block >= (int)((int64_t)blocks * (xcd + 1) >> 3)) return;
  const int row0 = block % p.nb_m * R::kRows, tile0 = block / p.nb_m * R::kTiles;
  const int last_row = p.M - 1 - row0, last_tile = p.n_tiles - 1 - tile0;
  const uint32_t lds0 = MDZ_LDS_ADDR(lds_raw);

  // A wave's loads of a turn: where the piece's memory begins, a lane's place in it, how far the next block is.  (Loads beyond the last piece repeat it;
  // rows beyond M repeat the last and tiles beyond the matrix its last: neither is stored.)  A lane of a piece of X has the 16-byte
  // chunk of its row that stands in its place: chunk c of row r is at c ^ (r % 16), so that 16 rows' chunks are read without bank conflicts.
  const uint8_t* base[L];
  uint32_t off[L], chunk[L];
  int step[L], dst[L];
  static_for<L>([&](auto i) {
    constexpr int q = decltype(i)::value;
    const int v = min(q * NW + wave, R::kPieces - 1);
    dst[q] = v * 1024;
    if (v < R::kX) {
      const int row = v * 4 + q4;
      base[q] = reinterpret_cast<const uint8_t*>(p.X) + (int64_t)row0 * p.ldx, step[q] = 2 * kI4Block;
      off[q] = (uint32_t)min(row, last_row) * (uint32_t)p.ldx, chunk[q] = (r16 ^ (row & 15)) * 16;
    } else {
      const int kind = v < R::kAtScales ? 0 : !ZEROS || v < R::kAtZeros ? 1 : 2, size = kind == 0 ? 1024 : kind == 1 ? 32 * G : 16 * G;
      const int c = v - (kind == 0 ? R::kX : kind == 1 ? R::kAtScales : R::kAtZeros), per = kind == 0 ? R::kTiles : kind == 1 ? R::kScales : max(R::kZeros, 1);
      const I4Matrix w = GATED && c >= per ? p.w[1] : p.w[0];
      const int at = c % per * 1024 + lane * 16, tile = min(min(at / size, R::kTiles - 1), last_tile);
      base[q] = (kind == 0 ? w.codes : kind == 1 ? w.scales : w.zeros) + (int64_t)tile0 * p.n_blocks * size, step[q] = size;
      off[q] = (uint32_t)tile * (uint32_t)p.n_blocks * (uint32_t)size + at % size, chunk[q] = 0;
    }
    base[q] = uniform(base[q]), step[q] = __builtin_amdgcn_readfirstlane(step[q]);
    dst[q] = __builtin_amdgcn_readfirstlane(dst[q]);
  });
  auto request = [&](int b) {
    const uint32_t slot = lds0 + b % 2 * R::kTurn;
    static_for<L>([&](auto i) {
      constexpr int q = decltype(i)::value;
      // (the last chunk again for those beyond K: a load stays inside its row; clear_behind_k)
      const uint32_t o = off[q] + min(chunk[q], (uint32_t)(p.K - 8 - b * kI4Block) * 2);
      load_to_lds<0>(base[q] + (uint32_t)(b * step[q]), o, slot + dst[q]);
    });
  };
  // Zeros in place of the chunks beyond K, in the pieces of X that this wave has loaded.  (The codes there are their zero points, but products with 16 + q and
  // what is taken off them cancel in exact arithmetic alone: with the last chunk up to sixteen times in the sums these lost four bits, and overflowed where all
  // that they stand for is far inside fp32's range.)
  auto clear_behind_k = [&](int b) {
    static_assert(R::kX % NW == 0, "a wave's first loads are its pieces of X");
    // (the lane's number made anew, from a zero that the compiler does not know: no register is held through the loop for it)
    uint32_t l = 0;
    asm volatile("" : "+v"(l));
    l = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, l));
#pragma unroll
    for (int q = 0; q < R::kX / NW; ++q) {
      const uint32_t v = q * NW + wave, row = v * 4 + (l >> 4), at = (l & 15) ^ (row & 15);
      if ((int)at * 8 >= p.K - b * kI4Block) *reinterpret_cast<u32x4_t*>(lds_raw + b % 2 * R::kTurn + v * 1024 + l * 16) = u32x4_t{0, 0, 0, 0};
    }
    wait_lds();
  };

  f32x4_t tot[NT][MT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MT; ++i) tot[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const I4Constants<E> constants;

  request(0);
  for (int b = 0; b < p.n_blocks; ++b) {
    wait_lds();
    wait_loads<0>();
    if ((b + 1) * kI4Block > p.K) clear_behind_k(b);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (b + 1 < p.n_blocks) request(b + 1);
    const uint8_t* const xs = lds_raw + b % 2 * R::kTurn;
    u32x4_t x[4][MT];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < MT; ++i)
        x[s][i] = *reinterpret_cast<const u32x4_t*>(xs + (i * 16 + r16) * 256 + (((s * 4 + q4) ^ r16) * 16));
    f32x4_t c0[G][MT];
    sum_block<E, G, ZEROS>(c0, x);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int mat = GATED && j >= NT / 2, tile = wave * (NT / R::kMats) + (GATED ? j % (NT / 2) : j);
      const uint8_t* const cs = xs + (R::kX + mat * R::kTiles + tile) * 1024 + lane * 16;
      const uint8_t* const ss = xs + (R::kAtScales + mat * R::kScales) * 1024 + tile * (32 * G) + q4 * (8 * G);
      I4Zeros<E, G> z{};
      if constexpr (ZEROS) z.load(xs + (R::kAtZeros + mat * R::kZeros) * 1024 + tile * (16 * G) + z.which(lane) * z.kStep);
      multiply_tile<E, G, ZEROS>(tot[j], x, c0, *reinterpret_cast<const u32x4_t*>(cs), *reinterpret_cast<const I4Scales<G>*>(ss), z, constants);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) asm volatile("" : "+v"(tot[j][i]));
  }
  finish_i4<E, GATED, MT, NT, 1>(p, tot, nullptr, row0, tile0 + wave * (NT / R::kMats), 0, lane);
}

template <typename E, int G, bool ZEROS, bool GATED, int MT, int NT, int XR, int NW, int D, int DX, int WPE>
static int launch_i4_few(I4Product p, hipStream_t st) {
  constexpr int kGateTiles = GATED ? NT / 2 : NT;
  constexpr int kLds = NW * 1024 * (XR > MT * NT ? XR : MT * NT);
  const int64_t columns = (p.n_tiles + kGateTiles - 1) / kGateTiles;
  MDZ_REQUIRE(columns * NW * 64 <= (int64_t)UINT32_MAX, MDZ_EUNSUPPORTED, "linear_i4: %d columns are more than one launch takes", p.N);
  auto kernel = gemm_i4_kernel<E, G, ZEROS, GATED, MT, NT, XR, NW, D, DX, WPE>;
  MDZ_SET_LDS_ONCE(kernel, kLds);
  launch_timed(PROF_GEMM_I4, kernel, dim3((unsigned)columns, (p.M + MT * 16 - 1) / (MT * 16)), NW * 64, kLds, st, p);
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

template <typename E, int G, bool ZEROS, bool GATED, int MT, int NT, int NW, int WPE>
static int launch_i4_rows(I4Product p, hipStream_t st) {
  typedef I4Ring<G, ZEROS, GATED, MT, NT, NW> R;
  static_assert(R::kLds <= 80 * 1024, "two workgroups share a CU's LDS");
  p.nb_m = (p.M + R::kRows - 1) / R::kRows, p.nb_n = (p.n_tiles + R::kTiles - 1) / R::kTiles;
  const int64_t workgroups = ((int64_t)p.nb_m * p.nb_n + 7) / 8 * 8;
  MDZ_REQUIRE(workgroups * NW * 64 <= (int64_t)UINT32_MAX, MDZ_EUNSUPPORTED, "linear_i4: %d x %d outputs are more than one launch takes", p.M, p.N);
  auto kernel = gemm_i4_rows_kernel<E, G, ZEROS, GATED, MT, NT, NW, WPE>;
  MDZ_SET_LDS_ONCE(kernel, R::kLds);
  launch_timed(PROF_GEMM_I4, kernel, dim3((unsigned)workgroups), NW * 64, R::kLds, st, p);
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

// few rows: rows / 16, tiles, pieces of X, waves; blocks of weights and of X requested ahead, waves per SIMD that the registers allow
// more rows: rows / 16 and tiles of a wave, waves, waves per SIMD
#define MDZ_I4_CASES                    \
  MDZ_I4_FEW(1, 1, 1, 8, 8, 8, 2)       \
  MDZ_I4_FEW(1, 2, 1, 8, 4, 4, 2)       \
  MDZ_I4_FEW(1, 2, 1, 4, 6, 6, 2)       \
  MDZ_I4_FEW(1, 4, 1, 4, 4, 4, 2)       \
  MDZ_I4_FEW(1, 1, 2, 8, 5, 5, 2)       \
  MDZ_I4_FEW(1, 2, 2, 8, 4, 4, 2)       \
  MDZ_I4_FEW(1, 2, 2, 4, 5, 5, 2)       \
  MDZ_I4_FEW(1, 4, 2, 4, 4, 4, 2)       \
  MDZ_I4_FEW(1, 1, 4, 8, 4, 4, 2)       \
  MDZ_I4_FEW(1, 2, 4, 8, 3, 3, 2)       \
  MDZ_I4_FEW(1, 2, 4, 4, 4, 4, 2)       \
  MDZ_I4_FEW(1, 4, 4, 4, 3, 3, 2)       \
  MDZ_I4_FEW(2, 1, 8, 8, 3, 1, 2)       \
  MDZ_I4_FEW(2, 2, 8, 8, 3, 1, 2)       \
  MDZ_I4_FEW(2, 6, 8, 4, 3, 1, 1)       \
  MDZ_I4_FEW(4, 1, 16, 8, 4, 1, 2)      \
  MDZ_I4_FEW(4, 2, 16, 8, 2, 1, 2)      \
  MDZ_I4_FEW(4, 6, 16, 4, 2, 1, 1)      \
  MDZ_I4_ROWS(4, 2, 4, 2)               \
  MDZ_I4_ROWS(4, 4, 4, 2)
template <typename E, int G, bool ZEROS, bool GATED>
static int launch_i4_tiles(const I4Product& p, const I4Plan& plan, hipStream_t st) {
  constexpr int kKind = i4_kind(__is_same(E, f16_t), G, ZEROS);
#define MDZ_I4_FEW(MT, NT, XR, NW, D, DX, WPE)                                                        \
  if constexpr ((!GATED || NT % 2 == 0) && i4_built(I4Plan{MT, NT, NW, XR}, kKind, GATED))             \
    if (plan.mt == MT && plan.nt == NT && plan.xr == XR && plan.waves == NW)                           \
      return launch_i4_few<E, G, ZEROS, GATED, MT, NT, XR, NW, D, DX, WPE>(p, st);
#define MDZ_I4_ROWS(MT, NT, NW, WPE) \
  if constexpr (i4_built(I4Plan{MT, NT, NW, 0}, kKind, GATED)) \
    if (plan.mt == MT && plan.nt == NT && plan.xr == 0 && plan.waves == NW) return launch_i4_rows<E, G, ZEROS, GATED, MT, NT, NW, WPE>(p, st);
  MDZ_I4_CASES
  MDZ_FAIL(MDZ_EINVAL, "linear_i4: no kernel of %d x %d tiles", plan.mt, plan.nt);
}

template <typename E, int G>
int launch_i4(const I4Product& p, bool zeros, bool gated, const I4Plan& plan, hipStream_t st) {
  if (zeros) return gated ? launch_i4_tiles<E, G, true, true>(p, plan, st) : launch_i4_tiles<E, G, true, false>(p, plan, st);
  return gated ? launch_i4_tiles<E, G, false, true>(p, plan, st) : launch_i4_tiles<E, G, false, false>(p, plan, st);
}

}  // namespace mdz
