// Sampling: one token per row of logits from a given random number, with a temperature, top-k, top-p and min-p (include/medusa.h, "sampling").
//
// Mathematics.  A token's mass is exp((logit - largest) / temperature), held as a 64-bit integer in units of 2^-S of the largest's (S = 62 less the bits
// of the vocabulary's size, at most 50): integer sums do not depend on the order of atomics, and a row's masses always fit.  In the order of the logits
// (descending, ties to the lower index) everything that is asked of a row is a place in one running sum: top-k the mass of the first k, top-p the first
// token up to which p of that lies, min-p the mass of the logits from a border on; the kept tokens are the shortest of these beginnings, and the draw is the
// token at which the running sum passes u times their mass.  So nothing is sorted but the bin of a histogram in which such a place lies.
//
// Bins: 1024 steps of (largest - logit) / temperature, 1/32 each.  A place is found in the bins' running sums; its bin is cut again, by 64ths of a bin or by the
// bits of its logits, until up to 64 tokens are left, which a wave sorts, or equal ones, which are counted.  Which bins the places of a row can
// lie in follows from the running sums alone, so their tokens are read once, into LDS (up to kCandidates; from memory each time beyond that).
//
// What bounds it.  A split row takes five launches that wait for each other: largest logit, histogram, ranges, their tokens, the draw; 1 x 128000 fp32 logits 3.0 + 5.9 +
// 5.5 + 4.4 + 6.6 us, all latency.  64 x 128000: 7.6 + 18.1 + 5.8 + 11.8 + 14.4; three passes over the logits, whose 33 MB take 7 us each, in the second the masses
// (6 us of 64-bit arithmetic: with masses of one instruction the pass took 12.6 of then 18.8 us, without sums over workgroups 18.0), in the
// fourth the wait for one addition per workgroup, in the last two passes over some 3000 candidates for each of two places.
#include "kernels.h"

namespace mdz {

constexpr int kBins = 1024;
constexpr float kBinsPerUnit = 32.f;
constexpr int kChunk = 4096;      // tokens that a workgroup has at a time where a row is split
constexpr int kSortMost = 64;     // tokens that a wave sorts
constexpr int kCandidates = 4096;  // tokens of the places' bins in LDS
constexpr uint32_t kTooMany = 1u << 30;  // (more than a vocabulary has)
constexpr int kMaskWords = kBins / 32;
constexpr int kChunkList = 256;   // chunks of a row whose masks are looked at together
constexpr int kCounterStep = 32;  // rows' counters of candidates stand in lines of their own: additions to one line wait for each other
// Up to here one wave settles a row faster than sixteen with barriers (us of a call at 1 x 128000 with 20 / 100 / 200 / 400 / 800 candidates: 24.0 / 25.8 / 27.9 /
// 31.8 / 38.1 by one wave, 25.6 / 26.0 / 26.7 / 28.0 / 30.1 by sixteen).
constexpr int kFewCandidates = 128;

struct BinRange {
  int first, last;
};
constexpr int kRanges = 4;

struct SampleArgs {
  const void* logits;
  int64_t ld;
  int rows, vocab, per, chunks, shift;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* token;
  float* prob;
  // Split rows.  Per row and chunk the largest logit and which bins it has tokens in; per row the histogram (then its running sums), the bins that its
  // places can be in, and their tokens.  span: chunks of a workgroup of the second pass.
  int span;
  float* chunk_max;
  uint32_t* mask;
  uint64_t* mass;
  uint64_t* candidate;
  uint32_t* count;
  uint32_t* candidates;
  BinRange* range;  // kRanges as find_ranges gives them, then the same without overlaps
  float* row_max;
};

// a row's settings, and the largest of its logits
struct RowSettings {
  float per_unit, largest, top;  // bins per unit of logits; top: the largest, or the largest number below plus infinity
  double rate;                   // log2(e) / temperature
  int top_k, shift;
  double top_p, min_p, u;
  __device__ inline RowSettings(const SampleArgs& a, int row) {
    const int s = row / a.per;
    const float t = a.temperature ? a.temperature[s] : 1.f;
    const bool greedy = !(t > 0.f);
    shift = a.shift;
    per_unit = greedy ? kBinsPerUnit : fminf(1.f / t * kBinsPerUnit, 3.402823466e38f);
    rate = greedy ? 1.4426950408889634 : 1.4426950408889634 / (double)t;
    top_k = greedy ? 1 : a.top_k ? a.top_k[s] : 0;
    top_p = a.top_p ? (double)a.top_p[s] : 1.0;
    min_p = a.min_p ? (double)a.min_p[s] : 0.0;
    u = (double)a.u[row];
  }
  __device__ inline void set_largest(float max) { largest = max, top = fminf(max, 3.402823466e38f); }
  // tokens that can be drawn: not NaN, not minus infinity; beside plus infinity nothing else
  __device__ inline bool valid(float l) const { return l > -INFINITY && (largest < INFINITY || l == largest); }
  // Monotone in l (a difference, a product and a conversion of fp32); what is not valid is somewhere among the bins too.
  __device__ inline int bin(float l) const { return (int)fmaxf(fminf((top - l) * per_unit, (float)(kBins - 1)), 0.f); }
  // 2^(shift + y), rounded to an integer; 2^f by its series, whose rest behind f^11 is below 7e-15, 9e-15 of 2^f (the masses' steps are 2^-45 at 128000 tokens).
  // y has four roundings (difference, log2(e), quotient, product), 4 * 2^-53 * 51 * ln 2 = 1.6e-14 of the mass where that is a step or more: 2^-45 with the series.
  __device__ inline uint64_t mass(float l) const {
    const double diff = (double)fminf(l, 3.402823466e38f) - (double)top;  // (zero for infinities beside an infinity)
    // (added to 1.5 * 2^52 a number is rounded to an integer, which the sum's low bits are)
    constexpr double kRound = 6755399441055744.0;
    const double y = fmax(diff * rate, -1000.0), at = y + kRound, f = y - (at - kRound);
    const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, at);
    double e = 4.4455382718708101e-10;
    e = fma(e, f, 7.0549116208011205e-09);
    e = fma(e, f, 1.0178086009239696e-07);
    e = fma(e, f, 1.3215486790144305e-06);
    e = fma(e, f, 1.5252733804059837e-05);
    e = fma(e, f, 1.5403530393381606e-04);
    e = fma(e, f, 1.3333558146428441e-03);
    e = fma(e, f, 9.6181291076284769e-03);
    e = fma(e, f, 5.5504108664821576e-02);
    e = fma(e, f, 2.4022650695910069e-01);
    e = fma(e, f, 6.9314718055994529e-01);
    e = fma(e, f, 1.0);
    // e * 2^(n + shift) to an integer, as above; -1000 + shift + 1023 is positive
    const double scale = __builtin_bit_cast(double, (uint64_t)(uint32_t)(n + shift + 1023) << 52);
    return __builtin_bit_cast(uint64_t, fma(e, scale, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
  }
};

// logit i of a row (minus zero as zero: they tie)
template <typename T>
__device__ inline float logit(const T* row, int i) { return to_float(row[i]) + 0.f; }
// The logits of a row from `at` on that fill 16 bytes, wherever the row starts; minus infinity behind the last.  (At a row's end the 16 bytes that end with
// it are loaded, so that there is one load and no branch, and many can be under way.)
template <typename T>
struct Some {
  static constexpr int kN = 16 / sizeof(T);
  u32x4_t raw;
  int from, at;
  __device__ inline Some() {}
  __device__ inline Some(const T* row, int at_, int vocab) : at(at_) {
    typedef u32x4_t Any __attribute__((aligned(2)));
    from = min(at, vocab - kN);
    if (vocab >= kN) {
      raw = *reinterpret_cast<const Any*>(row + from);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w = 0;
#pragma unroll
        for (int e = i * kN / 4; e < (i + 1) * kN / 4; ++e)
          if (from + e >= 0) {
            if constexpr (sizeof(T) == 4) w = __float_as_uint(row[from + e]);
            else w |= (uint32_t)row[from + e].bits << (16 * (e & 1));
          }
        raw[i] = w;
      }
    }
  }
  __device__ inline int index(int e) const { return from + e; }
  // (where the row is known not to end here)
  __device__ inline float inside(int e) const {
    const uint32_t w = raw[sizeof(T) == 4 ? e : e >> 1];
    if constexpr (sizeof(T) == 4) return __uint_as_float(w) + 0.f;
    else return to_float(T{(uint16_t)(e & 1 ? w >> 16 : w)}) + 0.f;
  }
  __device__ inline float operator[](int e) const { return from + e >= at ? inside(e) : -INFINITY; }
};
// as unsigned integers these order as the numbers do
__device__ inline uint32_t order_key(float l) {
  const uint32_t b = __float_as_uint(l);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <int NT, typename V, typename Op>
__device__ inline V block_reduce(V v, V* scratch, Op op) {  // scratch: NT / 64; the result in every thread
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = op(v, __shfl_xor(v, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  __syncthreads();
  v = scratch[0];
  for (int w = 1; w < NT / 64; ++w) v = op(v, scratch[w]);
  return v;
}

// ---- split rows: the first two passes ------------------------------------------------------------------
// The chunk's largest logit; the row's histogram is cleared on the way.
template <typename T>
__global__ void __launch_bounds__(256) sample_max_kernel(SampleArgs a) {
  __shared__ float scratch[4];
  const int chunk = blockIdx.x, row = blockIdx.y, first = chunk * kChunk;
  const T* const l = reinterpret_cast<const T*>(a.logits) + row * a.ld;
  constexpr int kN = Some<T>::kN;
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kChunk / 256 / kN; ++i) {
    const Some<T> x(l, first + (i * 256 + (int)threadIdx.x) * kN, a.vocab);
#pragma unroll
    for (int e = 0; e < kN; ++e) m = fmaxf(m, x[e]);
  }
  for (int b = chunk * 256 + (int)threadIdx.x; b < kBins; b += a.chunks * 256) {
    a.mass[(int64_t)row * kBins + b] = 0;
    a.count[(int64_t)row * kBins + b] = 0;
  }
  m = block_reduce<256>(m, scratch, [](float x, float y) { return fmaxf(x, y); });
  if (threadIdx.x == 0) a.chunk_max[(int64_t)row * a.chunks + chunk] = m;
}

template <int NT>
__device__ inline float row_max(const SampleArgs& a, int row, float* scratch) {
  float m = -INFINITY;
  for (int c = threadIdx.x; c < a.chunks; c += NT) m = fmaxf(m, a.chunk_max[(int64_t)row * a.chunks + c]);
  return block_reduce<NT>(m, scratch, [](float x, float y) { return fmaxf(x, y); });
}

// The tokens of a.span chunks into the row's histogram, through LDS, and which bins they are in.  A chunk is requested while the one before it is
// counted.
template <typename T>
__global__ void __launch_bounds__(256) sample_bins_kernel(SampleArgs a) {
  __shared__ uint64_t mass[kBins];
  __shared__ uint32_t count[kBins];
  __shared__ float scratch[4];
  const int row = blockIdx.y, chunk0 = blockIdx.x * a.span, chunks = min(a.span, a.chunks - chunk0);
  const T* const l = reinterpret_cast<const T*>(a.logits) + row * a.ld;
  constexpr int kN = Some<T>::kN, kLoads = kChunk / 256 / kN;
  Some<T> x[kLoads];
  auto load = [&](int chunk) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) x[i] = Some<T>(l, min(chunk * kChunk + (i * 256 + (int)threadIdx.x) * kN, a.vocab), a.vocab);
  };
  load(chunk0);
  for (int b = threadIdx.x; b < kBins; b += 256) mass[b] = 0, count[b] = 0;
  RowSettings s(a, row);
  s.set_largest(row_max<256>(a, row, scratch));
  for (int c = 0; c < chunks; ++c) {
    Some<T> now[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) now[i] = x[i];
    if (c + 1 < chunks) load(chunk0 + c + 1);
    auto add = [&](auto whole) {
#pragma unroll
      for (int i = 0; i < kChunk / 256; ++i) {
        const float v = decltype(whole)::value ? now[i / kN].inside(i % kN) : now[i / kN][i % kN];
        if (!s.valid(v)) continue;
        const int b = s.bin(v);
        atomicAdd((unsigned long long*)&mass[b], (unsigned long long)s.mass(v));
        atomicAdd(&count[b], 1u);
      }
    };
    if ((chunk0 + c + 1) * kChunk <= a.vocab) add(std::true_type{});
    else add(std::false_type{});
  }
  __syncthreads();
  for (int b = threadIdx.x; b < kBins; b += 256) {
    const uint32_t n = count[b];
    const uint64_t lanes = __ballot(n != 0);  // 64 bins: two words of the mask
    if ((threadIdx.x & 31) == 0)
      for (int c = 0; c < chunks; ++c)
        a.mask[((int64_t)row * a.chunks + chunk0 + c) * kMaskWords + (b >> 5)] = (uint32_t)(lanes >> (threadIdx.x & 32));
    if (n != 0) {
      atomicAdd((unsigned long long*)&a.mass[(int64_t)row * kBins + b], (unsigned long long)mass[b]);
      atomicAdd(&a.count[(int64_t)row * kBins + b], n);
    }
  }
}

// ---- the row's places -------------------------------------------------------------------------------------
// running sums of kBins counts and masses in LDS, in place
template <int NT>
__device__ inline void running_sums(uint64_t* mass, uint32_t* count, uint64_t* scratch) {  // scratch: 2 NT / 64
  constexpr int kPer = kBins / NT;
  static_assert(kPer >= 1 && kBins % NT == 0, "a thread has whole bins");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b0 = threadIdx.x * kPer;
  __syncthreads();
  uint64_t m[kPer];
  uint32_t c[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    m[i] = mass[b0 + i] + (i ? m[i - 1] : 0);
    c[i] = count[b0 + i] + (i ? c[i - 1] : 0);
  }
  uint64_t tm = m[kPer - 1];
  uint32_t tc = c[kPer - 1];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t om = __shfl_up((unsigned long long)tm, d);
    const uint32_t oc = __shfl_up(tc, d);
    if (lane >= d) tm += om, tc += oc;
  }
  if (lane == 63) scratch[2 * wave] = tm, scratch[2 * wave + 1] = tc;
  __syncthreads();
  tm -= m[kPer - 1], tc -= c[kPer - 1];
  for (int w = 0; w < wave; ++w) tm += scratch[2 * w], tc += (uint32_t)scratch[2 * w + 1];
#pragma unroll
  for (int i = 0; i < kPer; ++i) mass[b0 + i] = tm + m[i], count[b0 + i] = tc + c[i];
  __syncthreads();
}

struct Place {
  uint64_t through;  // mass of all tokens up to and with this one
  uint64_t mass;     // of the token
  int index;         // of the token, where it was asked for
};
enum PlaceOf { PLACE_OF_COUNT, PLACE_OF_MASS };  // the first token up to and with which the count, or the mass, is the target's

// The one workgroup that has a row, kRowThreads wide.
constexpr int kRowThreads = 1024;
struct RowLds {
  uint64_t mass[kBins];  // running sums of the row's histogram
  uint32_t count[kBins];
  uint64_t sub_mass[kBins];
  uint32_t sub_count[kBins];
  uint64_t candidate[kCandidates];  // key << 32 | index
  uint64_t list[kSortMost];         // ~key << 32 | index: sorted ascending these are the tokens in their order
  uint64_t through[kSortMost];
  uint64_t scratch[2 * kRowThreads / 64];
  float fscratch[kRowThreads / 64];
  uint32_t uscratch[kRowThreads / 64];
  uint32_t n, found, candidates, chunks_listed;
  uint16_t chunk[kChunkList];
  BinRange range[kRanges];
};
__device__ inline float key_logit(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }

// Calls f(logit, index) for the valid tokens of the bins of up to kRanges ranges, read from memory.  Of a split row only the chunks that have such tokens are
// read: their masks are looked at together, and the chunks' tokens then requested as one list.
template <typename T, typename F>
__device__ inline void for_ranges(const SampleArgs& a, const RowSettings& s, const T* l, int row, RowLds& d, const BinRange (&ranges)[kRanges], F&& f) {
  constexpr int NT = kRowThreads, kN = Some<T>::kN, kParts = kChunk / kN;
  int least = kBins, most = -1;
#pragma unroll
  for (int r = 0; r < kRanges; ++r)
    if (ranges[r].last >= ranges[r].first) least = min(least, ranges[r].first), most = max(most, ranges[r].last);
  for (int first = 0; first < a.chunks; first += kChunkList) {
    int n = min(a.chunks - first, kChunkList);
    if (a.mask) {
      __syncthreads();
      if (threadIdx.x == 0) d.chunks_listed = 0;
      __syncthreads();
      for (int c = threadIdx.x; c < n; c += NT) {
        const uint32_t* const m = a.mask + ((int64_t)row * a.chunks + first + c) * kMaskWords;
        uint32_t any = 0;
        for (const BinRange& r : ranges)
          for (int w = r.first >> 5; w <= r.last >> 5; ++w) {
            const uint32_t from = w == r.first >> 5 ? ~0u << (r.first & 31) : ~0u, to = w == r.last >> 5 ? ~0u >> (31 - (r.last & 31)) : ~0u;
            any |= m[w] & from & to;
          }
        if (any) d.chunk[atomicAdd(&d.chunks_listed, 1u)] = (uint16_t)c;
      }
      __syncthreads();
      n = (int)d.chunks_listed;
    }
    constexpr int kAhead = 4;  // loads under way
    const int total = n * kParts;
    for (int i0 = threadIdx.x; i0 < total; i0 += kAhead * NT) {
      Some<T> x[kAhead];
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        const int i = min(i0 + q * NT, total - 1), chunk = first + (a.mask ? d.chunk[i / kParts] : i / kParts);
        x[q] = Some<T>(l, min(chunk * kChunk + i % kParts * kN, a.vocab), a.vocab);
      }
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        if (i0 + q * NT >= total) break;
#pragma unroll
        for (int e = 0; e < kN; ++e) {
          const float v = x[q][e];
          const int b = s.bin(v);
          if (b < least || b > most) continue;  // (most tokens end here)
          bool in = false;
#pragma unroll
          for (int r = 0; r < kRanges; ++r) in |= b >= ranges[r].first && b <= ranges[r].last;
          if (in && s.valid(v)) f(v, x[q].index(e));
        }
      }
    }
  }
}
// the same for one range
template <typename T, typename F>
__device__ inline void for_bins(const SampleArgs& a, const RowSettings& s, const T* l, int row, RowLds& d, int b0, int b1, F&& f) {
  for_ranges(a, s, l, row, d, {{b0, b1}, {0, -1}, {0, -1}, {0, -1}}, f);
}

// the first of n running sums that reaches the target (the last, if none does); one thread finds it
template <typename Reached>
__device__ inline int first_reached(int n, uint32_t* found, Reached&& reached) {
  __syncthreads();
  if (threadIdx.x == 0) *found = n - 1;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kRowThreads)
    if (reached(i) && (i == 0 || !reached(i - 1))) *found = i;
  __syncthreads();
  return (int)*found;
}

// Requires 1 <= target <= the row's count or mass.  (Loops and the list are bounded by themselves, whatever becomes of the logits meanwhile.)
template <typename T>
__device__ inline Place find_place(const SampleArgs& a, const RowSettings& s, const T* l, int row, RowLds& d, PlaceOf of, uint64_t target, bool want_index) {
  constexpr int NT = kRowThreads;
  const int b = first_reached(kBins, &d.found, [&](int i) { return (of == PLACE_OF_COUNT ? (uint64_t)d.count[i] : d.mass[i]) >= target; });
  uint64_t before_mass = b ? d.mass[b - 1] : 0;
  uint32_t before_count = b ? d.count[b - 1] : 0, n = d.count[b] - before_count;
  uint32_t lo = 0, hi = 0xFFFFFFFFu;  // keys that are left of the bin
  for (int level = 0; n > kSortMost && level < 8; ++level) {
    uint32_t least = 0xFFFFFFFFu, most = 0;
    for_bins(a, s, l, row, d, b, b, [&](float v, int) {
      const uint32_t k = order_key(v);
      if (k >= lo && k <= hi) least = min(least, k), most = max(most, k);
    });
    least = block_reduce<NT>(least, d.uscratch, [](uint32_t x, uint32_t y) { return min(x, y); });
    most = block_reduce<NT>(most, d.uscratch, [](uint32_t x, uint32_t y) { return max(x, y); });
    if (least >= most) {  // all equal: the place is a matter of counting
      const uint64_t w = s.mass(key_logit(most));
      const uint64_t j = of == PLACE_OF_COUNT ? target - before_count - 1 : (target - before_mass + w - 1) / w - 1;
      Place p{before_mass + (j + 1) * w, w, -1};
      if (want_index) {  // the j-th of them by index: NT tokens at a time, counted in order
        if (threadIdx.x == 0) d.n = 0;
        uint64_t seen = 0;
        for (int first = 0; first < a.vocab && seen <= j; first += NT) {
          const int i = first + (int)threadIdx.x;
          const bool is = i < a.vocab && order_key(logit(l, i)) == most;
          const uint64_t lanes = __ballot(is);
          __syncthreads();
          if ((threadIdx.x & 63) == 0) d.uscratch[threadIdx.x >> 6] = (uint32_t)__popcll(lanes);
          __syncthreads();
          uint64_t mine = seen, all = 0;
          for (int w2 = 0; w2 < NT / 64; ++w2) {
            if (w2 < (int)(threadIdx.x >> 6)) mine += d.uscratch[w2];
            all += d.uscratch[w2];
          }
          mine += __popcll(lanes & ((1ull << (threadIdx.x & 63)) - 1));
          if (is && mine == j) d.n = (uint32_t)i;
          seen += all;
        }
        __syncthreads();
        p.index = (int)d.n;
      }
      return p;
    }
    // cut what is left by the keys' bits, the largest first
    const int shift = max(0, 32 - __clz(most - least) - 10);
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += NT) d.sub_mass[i] = 0, d.sub_count[i] = 0;
    __syncthreads();
    for_bins(a, s, l, row, d, b, b, [&](float v, int) {
      const uint32_t k = order_key(v);
      if (k < least || k > most) return;
      atomicAdd((unsigned long long*)&d.sub_mass[(most - k) >> shift], (unsigned long long)s.mass(v));
      atomicAdd(&d.sub_count[(most - k) >> shift], 1u);
    });
    running_sums<NT>(d.sub_mass, d.sub_count, d.scratch);
    const int c = first_reached(kBins, &d.found, [&](int i) {
      return (of == PLACE_OF_COUNT ? (uint64_t)before_count + d.sub_count[i] : before_mass + d.sub_mass[i]) >= target;
    });
    hi = most - ((uint32_t)c << shift);
    lo = max((uint64_t)least, (uint64_t)hi - min((uint64_t)hi, ((uint64_t)1 << shift) - 1));
    const uint64_t skipped = c ? d.sub_mass[c - 1] : 0;
    const uint32_t skipped_count = c ? d.sub_count[c - 1] : 0;
    n = d.sub_count[c] - skipped_count;
    before_mass += skipped, before_count += skipped_count;
  }
  n = min(n, (uint32_t)kSortMost);
  __syncthreads();
  if (threadIdx.x == 0) d.n = 0;
  __syncthreads();
  for_bins(a, s, l, row, d, b, b, [&](float v, int i) {
    const uint32_t k = order_key(v);
    if (k < lo || k > hi) return;
    const uint32_t at = atomicAdd(&d.n, 1u);
    if (at < n) d.list[at] = (uint64_t)~k << 32 | (uint32_t)i;
  });
  __syncthreads();
  if (threadIdx.x < 64) {  // each token's place is the number of those before it; then their running masses
    const bool is = threadIdx.x < n;
    const uint64_t mine = is ? d.list[threadIdx.x] : ~0ull;
    int before = 0;
    for (int i = 0; i < (int)n; ++i) before += __shfl((unsigned long long)mine, i) < mine;
    if (is) d.list[before] = mine;
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
    const uint64_t sorted = is ? d.list[threadIdx.x] : 0;
    uint64_t m = is ? s.mass(key_logit(~(uint32_t)(sorted >> 32))) : 0;
#pragma unroll
    for (int e = 1; e < 64; e <<= 1) {
      const uint64_t o = __shfl_up((unsigned long long)m, e);
      if ((int)threadIdx.x >= e) m += o;
    }
    if (is) d.through[threadIdx.x] = m;
  }
  const int j = first_reached((int)n, &d.found, [&](int i) {
    return (of == PLACE_OF_COUNT ? (uint64_t)before_count + i + 1 : before_mass + d.through[i]) >= target;
  });
  return Place{before_mass + d.through[j], d.through[j] - (j ? d.through[j - 1] : 0), (int)(uint32_t)d.list[j]};
}

// top-p: the mass that has to be reached; the draw: the one that the drawn token passes
__device__ inline uint64_t mass_for_p(double top_p, uint64_t mass) {
  const double p = ceil(fmax(top_p, 0.0) * (double)mass);
  return min(max((uint64_t)p, (uint64_t)1), mass);
}
__device__ inline uint64_t mass_for_u(double u, uint64_t kept) {
  const double at = u > 0.0 ? u * (double)kept : 0.0;
  return (at < (double)(kept - 1) ? (uint64_t)at : kept - 1) + 1;
}

// ---- the same by one wave, over candidates in LDS: no barriers ------------------------------------------------
__device__ inline void wave_order() {  // a wave's LDS accesses are done in order; this keeps the compiler's order
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}
template <typename V, typename Op>
__device__ inline V wave_reduce(V v, Op op) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = op(v, __shfl_xor(v, d));
  return v;
}
__device__ inline uint64_t wave_running_sum(uint64_t v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t o = __shfl_up((unsigned long long)v, d);
    if ((int)(threadIdx.x & 63) >= d) v += o;
  }
  return v;
}
// the first of the kBins running sums that reaches the target (the last, if none does): of 64 groups of 16, then of one
template <typename Reached>
__device__ inline int wave_first_bin(Reached&& reached) {
  const int lane = threadIdx.x & 63;
  const uint64_t groups = __ballot(reached(lane * 16 + 15));
  const int g = groups ? __builtin_ctzll(groups) : 63;
  const uint64_t bins = __ballot(lane < 16 && reached(g * 16 + (lane & 15)));
  return g * 16 + (bins ? __builtin_ctzll(bins) : 15);
}
// calls f(key, index, is) for the candidates, 64 at a time and in all lanes; `is`: of the bins and between the keys
template <typename F>
__device__ inline void for_candidates(const RowSettings& s, const RowLds& d, int b0, int b1, uint32_t lo, uint32_t hi, F&& f) {
  const int lane = threadIdx.x & 63, n = (int)d.candidates;
  for (int first = 0; first < n; first += 64) {
    const uint64_t c = d.candidate[min(first + lane, n - 1)];
    const uint32_t k = (uint32_t)(c >> 32);
    f(k, (uint32_t)c, first + lane < n && k >= lo && k <= hi && b0 <= s.bin(key_logit(k)) && s.bin(key_logit(k)) <= b1);
  }
}
__device__ inline Place wave_find_place(const RowSettings& s, RowLds& d, PlaceOf of, uint64_t target, bool want_index) {
  const int lane = threadIdx.x & 63;
  const int b = wave_first_bin([&](int i) { return (of == PLACE_OF_COUNT ? (uint64_t)d.count[i] : d.mass[i]) >= target; });
  uint64_t before_mass = b ? d.mass[b - 1] : 0;
  uint32_t before_count = b ? d.count[b - 1] : 0, n = d.count[b] - before_count;
  uint32_t lo = 0, hi = 0xFFFFFFFFu;
  for (int level = 0; n > kSortMost && level < 8; ++level) {
    uint32_t least = 0xFFFFFFFFu, most = 0;
    for_candidates(s, d, b, b, lo, hi, [&](uint32_t k, uint32_t, bool is) {
      if (is) least = min(least, k), most = max(most, k);
    });
    least = wave_reduce(least, [](uint32_t x, uint32_t y) { return min(x, y); });
    most = wave_reduce(most, [](uint32_t x, uint32_t y) { return max(x, y); });
    if (least >= most) {  // all equal: the place is a matter of counting
      const uint64_t w = s.mass(key_logit(most));
      const uint64_t j = of == PLACE_OF_COUNT ? target - before_count - 1 : (target - before_mass + w - 1) / w - 1;
      Place p{before_mass + (j + 1) * w, w, -1};
      if (want_index) {  // the least index up to which there are more than j of them, bit by bit
        uint32_t index = 0;
        for (int bit = 23; bit >= 0; --bit) {
          uint64_t below = 0;  // of those with the bits so far and a zero here, and all before them
          for_candidates(s, d, b, b, lo, hi, [&](uint32_t, uint32_t i, bool is) { below += __popcll(__ballot(is && i < (index | 1u << bit))); });
          if (below <= j) index |= 1u << bit;
        }
        p.index = (int)index;
      }
      return p;
    }
    const int shift = max(0, 32 - __clz(most - least) - 6);
    d.sub_mass[lane] = 0, d.sub_count[lane] = 0;
    wave_order();
    for_candidates(s, d, b, b, least, most, [&](uint32_t k, uint32_t, bool is) {
      if (!is) return;
      atomicAdd((unsigned long long*)&d.sub_mass[(most - k) >> shift], (unsigned long long)s.mass(key_logit(k)));
      atomicAdd(&d.sub_count[(most - k) >> shift], 1u);
    });
    wave_order();
    const uint64_t m = wave_running_sum(d.sub_mass[lane]), c = wave_running_sum(d.sub_count[lane]);
    const uint64_t at = __ballot((of == PLACE_OF_COUNT ? before_count + c : before_mass + m) >= target);
    const int i = at ? __builtin_ctzll(at) : 63;
    hi = most - ((uint32_t)i << shift);
    lo = max((uint64_t)least, (uint64_t)hi - min((uint64_t)hi, ((uint64_t)1 << shift) - 1));
    const uint64_t skipped = i ? __shfl((unsigned long long)m, i - 1) : 0, skipped_count = i ? __shfl((unsigned long long)c, i - 1) : 0;
    n = (uint32_t)(__shfl((unsigned long long)c, i) - skipped_count);
    before_mass += skipped, before_count += (uint32_t)skipped_count;
    wave_order();
  }
  n = min(n, (uint32_t)kSortMost);
  int listed = 0;
  for_candidates(s, d, b, b, lo, hi, [&](uint32_t k, uint32_t i, bool is) {
    const uint64_t lanes = __ballot(is);
    const int at = listed + __popcll(lanes & ((1ull << lane) - 1));
    if (is && at < (int)n) d.list[at] = (uint64_t)~k << 32 | i;
    listed += __popcll(lanes);
  });
  wave_order();
  const bool is = lane < (int)n;
  const uint64_t mine = is ? d.list[lane] : ~0ull;
  int before = 0;
  for (int i = 0; i < (int)n; ++i) {
    const uint32_t high = (uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), i), low = (uint32_t)__builtin_amdgcn_readlane((int)mine, i);
    before += ((uint64_t)high << 32 | low) < mine;
  }
  wave_order();
  if (is) d.list[before] = mine;
  wave_order();
  const uint64_t sorted = is ? d.list[lane] : 0, own = is ? s.mass(key_logit(~(uint32_t)(sorted >> 32))) : 0, m = wave_running_sum(own);
  const uint64_t at = __ballot(is && (of == PLACE_OF_COUNT ? (uint64_t)before_count + lane + 1 : before_mass + m) >= target);
  const int j = at ? __builtin_ctzll(at) : (int)n - 1;
  wave_order();
  return Place{before_mass + __shfl((unsigned long long)m, j), __shfl((unsigned long long)own, j), (int)(uint32_t)__shfl((unsigned long long)sorted, j)};
}

// ---- the same by all waves, over many candidates in LDS -------------------------------------------------------
// Calls f(key, index) for the candidates of a bin in the thread that has them.
template <typename F>
__device__ inline void block_candidates(const RowSettings& s, const RowLds& d, int b0, int b1, F&& f) {
  for (int i = threadIdx.x, n = (int)d.candidates; i < n; i += kRowThreads) {
    const uint64_t c = d.candidate[i];
    const int b = s.bin(key_logit((uint32_t)(c >> 32)));
    if (b >= b0 && b <= b1) f((uint32_t)(c >> 32), (uint32_t)c);
  }
}
// The bin is cut once more by the same steps, 1/64 of a bin each; the tokens of the 64th in which the place lies are sorted, by every wave for itself.  (More than
// a wave has lanes: ties, or nearly; wave_find_place cuts those by their bits.)
__device__ inline Place block_find_place(const RowSettings& s, RowLds& d, PlaceOf of, uint64_t target, bool want_index) {
  const int lane = threadIdx.x & 63;
  const int b = wave_first_bin([&](int i) { return (of == PLACE_OF_COUNT ? (uint64_t)d.count[i] : d.mass[i]) >= target; });
  uint64_t before_mass = b ? d.mass[b - 1] : 0;
  uint32_t before_count = b ? d.count[b - 1] : 0;
  if (threadIdx.x < 64) d.sub_mass[lane] = 0, d.sub_count[lane] = 0;
  if (threadIdx.x == 0) d.n = 0;
  __syncthreads();
  // monotone as the bins are: of the same fp32 number
  auto part = [&](uint32_t k) { return (int)fmaxf(fminf(((s.top - key_logit(k)) * s.per_unit - (float)b) * 64.f, 63.f), 0.f); };
  block_candidates(s, d, b, b, [&](uint32_t k, uint32_t) {
    atomicAdd((unsigned long long*)&d.sub_mass[part(k)], (unsigned long long)s.mass(key_logit(k)));
    atomicAdd(&d.sub_count[part(k)], 1u);
  });
  __syncthreads();
  const uint64_t sm = wave_running_sum(d.sub_mass[lane]), sc = wave_running_sum(d.sub_count[lane]);
  const uint64_t reached = __ballot((of == PLACE_OF_COUNT ? before_count + sc : before_mass + sm) >= target);
  const int i = reached ? __builtin_ctzll(reached) : 63;
  const uint64_t skipped_mass = i ? __shfl((unsigned long long)sm, i - 1) : 0, skipped = i ? __shfl((unsigned long long)sc, i - 1) : 0;
  const uint32_t n = (uint32_t)(__shfl((unsigned long long)sc, i) - skipped);
  if (n > kSortMost) {
    Place p{0, 0, -1};
    __syncthreads();
    if (threadIdx.x < 64) {
      p = wave_find_place(s, d, of, target, want_index);
      if (lane == 0) d.through[0] = p.through, d.through[1] = p.mass, d.through[2] = (uint64_t)(uint32_t)p.index;
    }
    __syncthreads();
    p = Place{d.through[0], d.through[1], (int)(uint32_t)d.through[2]};
    __syncthreads();
    return p;
  }
  before_mass += skipped_mass, before_count += (uint32_t)skipped;
  block_candidates(s, d, b, b, [&](uint32_t k, uint32_t index) {
    if (part(k) != i) return;
    const uint32_t at = atomicAdd(&d.n, 1u);
    if (at < n) d.list[at] = (uint64_t)~k << 32 | index;
  });
  __syncthreads();
  const bool is = lane < (int)n;
  const uint64_t mine = is ? d.list[lane] : ~0ull;
  int before = 0;
  for (int e = 0; e < (int)n; ++e) {
    const uint32_t high = (uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), e), low = (uint32_t)__builtin_amdgcn_readlane((int)mine, e);
    before += ((uint64_t)high << 32 | low) < mine;
  }
  const int to = (is ? before : lane) * 4;  // each lane's token to the lane of its place
  const uint32_t high = (uint32_t)__builtin_amdgcn_ds_permute(to, (int)(mine >> 32)), low = (uint32_t)__builtin_amdgcn_ds_permute(to, (int)mine);
  const uint64_t own = is ? s.mass(key_logit(~high)) : 0, m = wave_running_sum(own);
  const uint64_t at = __ballot(is && (of == PLACE_OF_COUNT ? (uint64_t)before_count + lane + 1 : before_mass + m) >= target);
  const int j = at ? __builtin_ctzll(at) : (int)n - 1;
  return Place{before_mass + __shfl((unsigned long long)m, j), __shfl((unsigned long long)own, j), __shfl((int)low, j)};
}

// ---- a row from its histogram to its token -----------------------------------------------------------------
// which cuts a row has, and the logit from which on tokens pass min-p: mass >= min_p  <=>  logit >= largest + temperature ln(min_p)
struct Cuts {
  bool by_k, by_p, by_min;
  double border;
  __device__ inline Cuts(const RowSettings& s, uint32_t tokens) {
    by_k = s.top_k > 0 && (uint32_t)s.top_k < tokens, by_p = s.top_p < 1.0;
    by_min = s.min_p > 0.0 && s.largest < INFINITY && s.rate > 0.0;  // (at an infinite temperature all masses are the largest)
    border = by_min ? (double)s.largest + log2(fmin(s.min_p, 1.0)) / s.rate : 0.0;
  }
};

// One wave, from the histogram's running sums: the bins that the places can be in, what is kept being known to within a bin at each cut.  Returns how many
// tokens they hold (ranges may overlap: at most).
__device__ inline uint32_t find_ranges(const RowSettings& s, const Cuts& cuts, const uint64_t* mass, const uint32_t* count, BinRange (&ranges)[kRanges]) {
  const uint64_t all = mass[kBins - 1];
  auto before = [&](int b) { return b ? mass[b - 1] : (uint64_t)0; };
  auto bin_of_mass = [&](uint64_t m) { return wave_first_bin([&](int i) { return mass[i] >= m; }); };
#pragma unroll
  for (int i = 0; i < kRanges; ++i) ranges[i] = BinRange{0, -1};
  uint64_t low = all, high = all;
  if (cuts.by_k) {
    const int b = wave_first_bin([&](int i) { return count[i] >= (uint32_t)s.top_k; });
    ranges[0] = {b, b}, low = max(before(b), (uint64_t)1), high = mass[b];
  }
  if (cuts.by_p) {
    const int b0 = bin_of_mass(mass_for_p(s.top_p, low)), b1 = low == high ? b0 : bin_of_mass(mass_for_p(s.top_p, high));
    ranges[1] = {b0, b1}, low = max(before(b0), (uint64_t)1), high = min(high, mass[b1]);
  }
  if (cuts.by_min) {  // (the border's rounding to fp32 may cross a bin)
    const int b = s.bin(fminf(fmaxf((float)cuts.border, -3.402823466e38f), s.largest));
    ranges[2] = {max(0, b - 1), min(kBins - 1, b + 1)};
    low = min(low, max(before(ranges[2].first), (uint64_t)1)), high = min(high, mass[ranges[2].last]);
  }
  const int b0 = bin_of_mass(mass_for_u(s.u, low)), b1 = low == high ? b0 : bin_of_mass(mass_for_u(s.u, high));
  ranges[3] = {b0, b1};
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kRanges; ++i)
    if (ranges[i].last >= ranges[i].first) most += count[ranges[i].last] - (ranges[i].first ? count[ranges[i].first - 1] : 0);
  return most;
}
__device__ inline bool in_ranges(const BinRange (&ranges)[kRanges], int b) {
  bool in = false;
#pragma unroll
  for (int i = 0; i < kRanges; ++i) in |= b >= ranges[i].first && b <= ranges[i].last;
  return in;
}

// d: the running sums and, if they are no more than kCandidates, the candidates.  All threads; the first writes the row's answer.
template <typename T>
__device__ inline void settle_row(const SampleArgs& a, const RowSettings& s, const T* l, int row, RowLds& d, const BinRange& min_range) {
  const Cuts cuts(s, d.count[kBins - 1]);
  const uint64_t before_min = min_range.first > 0 ? d.mass[min_range.first - 1] : 0;
  uint64_t kept = d.mass[kBins - 1];
  Place p;
  if (d.candidates > kFewCandidates && d.candidates <= kCandidates) {
    if (cuts.by_k) kept = block_find_place(s, d, PLACE_OF_COUNT, (uint64_t)s.top_k, false).through;
    if (cuts.by_p) kept = block_find_place(s, d, PLACE_OF_MASS, mass_for_p(s.top_p, kept), false).through;
    if (cuts.by_min) {
      unsigned long long mass = 0;
      block_candidates(s, d, min_range.first, min_range.last, [&](uint32_t k, uint32_t) {
        if ((double)key_logit(k) >= cuts.border) mass += s.mass(key_logit(k));
      });
      mass = block_reduce<kRowThreads>(mass, (unsigned long long*)d.scratch, [](unsigned long long x, unsigned long long y) { return x + y; });
      kept = min(kept, max(before_min + mass, (uint64_t)1 << s.shift));
    }
    p = block_find_place(s, d, PLACE_OF_MASS, mass_for_u(s.u, kept), true);
  } else if (d.candidates <= kCandidates) {
    if (threadIdx.x >= 64) return;
    if (cuts.by_k) kept = wave_find_place(s, d, PLACE_OF_COUNT, (uint64_t)s.top_k, false).through;
    if (cuts.by_p) kept = wave_find_place(s, d, PLACE_OF_MASS, mass_for_p(s.top_p, kept), false).through;
    if (cuts.by_min) {
      unsigned long long mass = 0;
      for_candidates(s, d, min_range.first, min_range.last, 0, 0xFFFFFFFFu, [&](uint32_t k, uint32_t, bool is) {
        if (is && (double)key_logit(k) >= cuts.border) mass += s.mass(key_logit(k));
      });
      mass = wave_reduce(mass, [](unsigned long long x, unsigned long long y) { return x + y; });
      kept = min(kept, max(before_min + mass, (uint64_t)1 << s.shift));
    }
    p = wave_find_place(s, d, PLACE_OF_MASS, mass_for_u(s.u, kept), true);
  } else {
    if (cuts.by_k) kept = find_place(a, s, l, row, d, PLACE_OF_COUNT, (uint64_t)s.top_k, false).through;
    if (cuts.by_p) kept = find_place(a, s, l, row, d, PLACE_OF_MASS, mass_for_p(s.top_p, kept), false).through;
    if (cuts.by_min) {
      unsigned long long mass = 0;
      for_bins(a, s, l, row, d, min_range.first, min_range.last, [&](float v, int) {
        if ((double)v >= cuts.border) mass += s.mass(v);
      });
      mass = block_reduce<kRowThreads>(mass, (unsigned long long*)d.scratch, [](unsigned long long x, unsigned long long y) { return x + y; });
      kept = min(kept, max(before_min + mass, (uint64_t)1 << s.shift));
    }
    p = find_place(a, s, l, row, d, PLACE_OF_MASS, mass_for_u(s.u, kept), true);
  }
  if (threadIdx.x == 0) {
    a.token[row] = p.index;
    if (a.prob) a.prob[row] = (float)((double)p.mass / (double)kept);
  }
}
__device__ inline void nothing_to_draw(const SampleArgs& a, int row) {
  if (threadIdx.x == 0) {
    a.token[row] = -1;
    if (a.prob) a.prob[row] = 0.f;
  }
}

// Split rows, third pass: a workgroup makes the running sums of a row's histogram and finds its ranges.
__global__ void __launch_bounds__(256) sample_ranges_kernel(SampleArgs a) {
  __shared__ uint64_t mass[kBins];
  __shared__ uint32_t count[kBins];
  __shared__ uint64_t sums[8];
  __shared__ float scratch[4];
  const int row = blockIdx.x;
  RowSettings s(a, row);
#pragma unroll
  for (int i = 0; i < kBins / 256; ++i) {
    const int b = i * 256 + (int)threadIdx.x;
    mass[b] = a.mass[(int64_t)row * kBins + b], count[b] = a.count[(int64_t)row * kBins + b];
  }
  s.set_largest(row_max<256>(a, row, scratch));
  running_sums<256>(mass, count, sums);
#pragma unroll
  for (int i = 0; i < kBins / 256; ++i) {
    const int b = i * 256 + (int)threadIdx.x;
    a.mass[(int64_t)row * kBins + b] = mass[b], a.count[(int64_t)row * kBins + b] = count[b];
  }
  if (threadIdx.x >= 64) return;
  BinRange ranges[kRanges] = {{0, -1}, {0, -1}, {0, -1}, {0, -1}};
  uint32_t most = 0;
  if (count[kBins - 1] != 0) most = find_ranges(s, Cuts(s, count[kBins - 1]), mass, count, ranges);
  if (threadIdx.x == 0) {
    const bool few = most <= 4 * kCandidates;
    a.candidates[row * kCounterStep] = few ? 0 : kTooMany;  // (then nobody gathers)
#pragma unroll
    for (int i = 0; i < kRanges; ++i) a.range[row * 2 * kRanges + i] = ranges[i];
    // ranges that touch become one (what stays over after these rounds is looked at twice, no more)
#pragma unroll
    for (int round = 0; round < 2; ++round)
#pragma unroll
      for (int i = 0; i < kRanges; ++i)
#pragma unroll
        for (int j = i + 1; j < kRanges; ++j) {
          BinRange &x = ranges[i], &y = ranges[j];
          if (y.first > y.last || (x.first <= x.last && (x.first > y.last + 1 || y.first > x.last + 1))) continue;
          x = x.first > x.last ? y : BinRange{min(x.first, y.first), max(x.last, y.last)}, y = {0, -1};
        }
#pragma unroll
    for (int i = 0; i < kRanges; ++i) a.range[row * 2 * kRanges + kRanges + i] = ranges[i];
    a.row_max[row] = s.largest;
  }
}

// Fourth pass: a chunk's tokens of the row's ranges to its candidates.
template <typename T>
__global__ void __launch_bounds__(256) sample_gather_kernel(SampleArgs a) {
  __shared__ uint32_t of_wave[4], first;
  const int chunk = blockIdx.x, row = blockIdx.y, lane = threadIdx.x & 63, first_of_chunk = chunk * kChunk;
  const T* const l = reinterpret_cast<const T*>(a.logits) + row * a.ld;
  constexpr int kN = Some<T>::kN, kLoads = kChunk / 256 / kN;
  Some<T> x[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) x[i] = Some<T>(l, min(chunk * kChunk + (i * 256 + (int)threadIdx.x) * kN, a.vocab), a.vocab);
  if (a.candidates[row * kCounterStep] >= kTooMany) return;
  BinRange ranges[kRanges];
#pragma unroll
  for (int i = 0; i < kRanges; ++i) ranges[i] = a.range[row * 2 * kRanges + kRanges + i];
  RowSettings s(a, row);
  s.set_largest(a.row_max[row]);
  constexpr int kOf = kLoads * kN;
  uint64_t is[kOf];  // which lanes' logits, each logit of a thread
  // A bin is the integer part of (top - logit) * per_unit but for the last one's and for infinities: where neither is near, the ranges' ends are compared with
  // that, and what cannot be drawn is above all of them, or not a number.
  bool plain = s.largest < INFINITY && s.per_unit > 0.f && first_of_chunk + kChunk <= a.vocab;
#pragma unroll
  for (int r = 0; r < kRanges; ++r) plain &= ranges[r].last < kBins - 1;
  if (plain) {
    float at[kOf];
#pragma unroll
    for (int k = 0; k < kOf; ++k) at[k] = (s.top - x[k / kN].inside(k % kN)) * s.per_unit, is[k] = 0;
#pragma unroll
    for (int r = 0; r < kRanges; ++r) {
      if (ranges[r].first > ranges[r].last) continue;
      const float from = (float)ranges[r].first, to = (float)(ranges[r].last + 1);
#pragma unroll
      for (int k = 0; k < kOf; ++k) is[k] |= __ballot(at[k] >= from) & __ballot(at[k] < to);
    }
  } else {
#pragma unroll
    for (int k = 0; k < kOf; ++k) is[k] = __ballot(in_ranges(ranges, s.bin(x[k / kN][k % kN])) && s.valid(x[k / kN][k % kN]));
  }
  uint32_t mine = 0;  // of the wave
#pragma unroll
  for (int k = 0; k < kOf; ++k) mine += __popcll(is[k]);
  // (one addition to the row's count per workgroup: they wait for each other; one per wave made 64 flat rows of 128000 take 39 us)
  if (lane == 0) of_wave[threadIdx.x >> 6] = mine;
  __syncthreads();
  const uint32_t all = of_wave[0] + of_wave[1] + of_wave[2] + of_wave[3];
  if (all == 0) return;
  if (threadIdx.x == 0) first = atomicAdd(&a.candidates[row * kCounterStep], all);
  __syncthreads();
  uint32_t at = first;
  for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) at += of_wave[w];
#pragma unroll
  for (int k = 0; k < kOf; ++k) {
    if (is[k] == 0) continue;
    const uint32_t to = at + __popcll(is[k] & ((1ull << lane) - 1));
    if ((is[k] >> lane & 1) && to < kCandidates)
      a.candidate[(int64_t)row * kCandidates + to] = (uint64_t)order_key(x[k / kN][k % kN]) << 32 | (uint32_t)x[k / kN].index(k % kN);
    at += __popcll(is[k]);
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) sample_draw_kernel(SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds_raw[];
  RowLds& d = *reinterpret_cast<RowLds*>(lds_raw);
  const int row = blockIdx.x;
  for (int b = threadIdx.x; b < kBins; b += kRowThreads) d.mass[b] = a.mass[(int64_t)row * kBins + b], d.count[b] = a.count[(int64_t)row * kBins + b];
  const uint32_t candidates = a.candidates[row * kCounterStep];
  if (candidates <= kCandidates)
    for (uint32_t i = threadIdx.x; i < candidates; i += kRowThreads) d.candidate[i] = a.candidate[(int64_t)row * kCandidates + i];
  if (threadIdx.x == 0) d.candidates = candidates;
  RowSettings s(a, row);
  s.set_largest(a.row_max[row]);
  __syncthreads();
  if (d.count[kBins - 1] == 0) return nothing_to_draw(a, row);
  settle_row(a, s, reinterpret_cast<const T*>(a.logits) + row * a.ld, row, d, a.range[row * 2 * kRanges + 2]);
}

// A row to a workgroup: all passes.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) sample_row_kernel(SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds_raw[];
  RowLds& d = *reinterpret_cast<RowLds*>(lds_raw);
  const int row = blockIdx.x;
  const T* const l = reinterpret_cast<const T*>(a.logits) + row * a.ld;
  float m = -INFINITY;
  constexpr int kN = Some<T>::kN;
#pragma unroll 4
  for (int i = threadIdx.x * kN; i < a.vocab; i += kRowThreads * kN) {
    const Some<T> x(l, i, a.vocab);
#pragma unroll
    for (int e = 0; e < kN; ++e) m = fmaxf(m, x[e]);
  }
  for (int b = threadIdx.x; b < kBins; b += kRowThreads) d.mass[b] = 0, d.count[b] = 0;
  RowSettings s(a, row);
  s.set_largest(block_reduce<kRowThreads>(m, d.fscratch, [](float x, float y) { return fmaxf(x, y); }));
#pragma unroll 2
  for (int i = threadIdx.x * kN; i < a.vocab; i += kRowThreads * kN) {
    const Some<T> x(l, i, a.vocab);
#pragma unroll
    for (int e = 0; e < kN; ++e) {
      const float v = x[e];
      if (!s.valid(v)) continue;
      const int b = s.bin(v);
      atomicAdd((unsigned long long*)&d.mass[b], (unsigned long long)s.mass(v));
      atomicAdd(&d.count[b], 1u);
    }
  }
  running_sums<kRowThreads>(d.mass, d.count, d.scratch);
  if (d.count[kBins - 1] == 0) return nothing_to_draw(a, row);
  if (threadIdx.x < 64) {
    BinRange ranges[kRanges];
    const uint32_t most = find_ranges(s, Cuts(s, d.count[kBins - 1]), d.mass, d.count, ranges);
    if (threadIdx.x == 0) {
#pragma unroll
      for (int i = 0; i < kRanges; ++i) d.range[i] = ranges[i];
      d.candidates = most <= 4 * kCandidates ? 0 : kCandidates + 1;
    }
  }
  __syncthreads();
  BinRange ranges[kRanges];
#pragma unroll
  for (int i = 0; i < kRanges; ++i) ranges[i] = d.range[i];
  const bool gather = d.candidates == 0;
  __syncthreads();
  if (gather)
    for_ranges(a, s, l, row, d, ranges, [&](float v, int i) {
      const uint32_t at = atomicAdd(&d.candidates, 1u);
      if (at < kCandidates) d.candidate[at] = (uint64_t)order_key(v) << 32 | (uint32_t)i;
    });
  __syncthreads();
  settle_row(a, s, l, row, d, ranges[2]);
}

// ---- the call ----------------------------------------------------------------------------------------------
constexpr int kMaxVocab = 1 << 24;  // the masses then still have 38 bits behind the point
static bool sample_splits(int rows, int vocab) { return vocab > 2 * kChunk && rows < num_cus(); }
// scratch of a call
static int64_t sample_bytes(int rows, int vocab) {
  if (!sample_splits(rows, vocab)) return 0;
  const int64_t chunks = (vocab + kChunk - 1) / kChunk;
  return rows * (kBins * 12 + kCandidates * 8 + 2 * kRanges * 8 + kCounterStep * 4 + 4 + chunks * (kMaskWords * 4 + 4));
}
// chunks of a workgroup of the second pass
static int sample_span(int rows, int chunks) {
  return (int64_t)rows * chunks > 4 * num_cus() ? 2 : 1;
}
static int check_sample(int rows, int vocab) {
  MDZ_REQUIRE(rows >= 0 && vocab > 0, MDZ_EINVAL, "sample: %d rows of %d logits", rows, vocab);
  MDZ_REQUIRE(vocab <= kMaxVocab && rows <= 1 << 21, MDZ_EUNSUPPORTED, "sample: up to 2^21 rows of 2^24 logits (%d of %d)", rows, vocab);
  return MDZ_OK;
}

template <typename T>
static int launch_sample(const SampleArgs& a, bool split, hipStream_t st) {
  if (!split) {
    MDZ_SET_LDS_ONCE(sample_row_kernel<T>, sizeof(RowLds));
    launch_timed(PROF_SELECT, sample_row_kernel<T>, (unsigned)a.rows, kRowThreads, sizeof(RowLds), st, a);
    MDZ_LAUNCH_CHECK();
    return MDZ_OK;
  }
  MDZ_SET_LDS_ONCE(sample_draw_kernel<T>, sizeof(RowLds));
  launch_timed(PROF_SELECT, sample_max_kernel<T>, dim3(a.chunks, a.rows), 256, 0, st, a);
  MDZ_LAUNCH_CHECK();
  launch_timed(PROF_SELECT, sample_bins_kernel<T>, dim3((a.chunks + a.span - 1) / a.span, a.rows), 256, 0, st, a);
  MDZ_LAUNCH_CHECK();
  launch_timed(PROF_SELECT, sample_ranges_kernel, (unsigned)a.rows, 256, 0, st, a);
  MDZ_LAUNCH_CHECK();
  launch_timed(PROF_SELECT, sample_gather_kernel<T>, dim3(a.chunks, a.rows), 256, 0, st, a);
  MDZ_LAUNCH_CHECK();
  launch_timed(PROF_SELECT, sample_draw_kernel<T>, (unsigned)a.rows, kRowThreads, sizeof(RowLds), st, a);
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

}  // namespace mdz

using namespace mdz;

extern "C" {
#pragma GCC visibility push(default)

int64_t medusa_sample_workspace_bytes(int rows, int vocab) {
  const int rc = check_sample(rows, vocab);
  // (of the call of up to so many rows that needs most: one of many more, whose rows are not split, needs none itself)
  return rc ? rc : sample_bytes(rows < num_cus() ? rows : num_cus() - 1, vocab);
}

int medusa_sample(int dtype, const void* logits, int64_t ld, int rows, int vocab, const float* temperature_opt, const int32_t* top_k_opt,
                  const float* top_p_opt, const float* min_p_opt, int rows_per_setting, const float* u, int32_t* token, float* prob_opt, void* ws,
                  int64_t ws_bytes, void* stream) {
  MDZ_REQUIRE(dtype_ok(dtype), MDZ_EINVAL, "sample: bad dtype %d", dtype);
  const int rc = check_sample(rows, vocab);
  if (rc) return rc;
  MDZ_REQUIRE(rows_per_setting > 0, MDZ_EINVAL, "sample: %d rows per setting", rows_per_setting);
  MDZ_REQUIRE(ld >= vocab, MDZ_ESHAPE, "sample: rows %lld apart hold %d logits", (long long)ld, vocab);
  if (rows == 0) return MDZ_OK;
  MDZ_REQUIRE(logits && u && token, MDZ_EINVAL, "sample: NULL pointer");
  const uintptr_t four = reinterpret_cast<uintptr_t>(temperature_opt) | reinterpret_cast<uintptr_t>(top_k_opt) | reinterpret_cast<uintptr_t>(top_p_opt) |
                         reinterpret_cast<uintptr_t>(min_p_opt) | reinterpret_cast<uintptr_t>(u) | reinterpret_cast<uintptr_t>(token) |
                         reinterpret_cast<uintptr_t>(prob_opt);
  MDZ_REQUIRE(four % 4 == 0 && reinterpret_cast<uintptr_t>(logits) % elem_bytes(dtype) == 0, MDZ_EINVAL, "sample: a buffer is not aligned to its elements");
  const int64_t need = sample_bytes(rows, vocab);
  MDZ_REQUIRE(ws_bytes >= need && (ws || need == 0), MDZ_EWORKSPACE, "sample: workspace %lld < %lld bytes", (long long)ws_bytes, (long long)need);
  MDZ_REQUIRE(need == 0 || reinterpret_cast<uintptr_t>(ws) % 16 == 0, MDZ_EINVAL, "sample: the workspace must start on 16 bytes");
  SampleArgs a{};
  a.logits = logits, a.ld = ld, a.rows = rows, a.vocab = vocab, a.per = rows_per_setting, a.chunks = (vocab + kChunk - 1) / kChunk;
  int bits = 0;
  while ((int64_t)1 << bits < vocab) ++bits;
  a.shift = 62 - bits < 50 ? 62 - bits : 50;
  a.temperature = temperature_opt, a.top_k = top_k_opt, a.top_p = top_p_opt, a.min_p = min_p_opt, a.u = u, a.token = token, a.prob = prob_opt;
  const bool split = need != 0;
  if (split) {
    const int64_t n = rows, chunks = a.chunks;
    a.span = sample_span(rows, a.chunks);
    a.mass = (uint64_t*)ws, a.candidate = a.mass + n * kBins;
    a.range = (BinRange*)(a.candidate + n * kCandidates);
    a.count = (uint32_t*)(a.range + n * 2 * kRanges), a.candidates = a.count + n * kBins;
    a.mask = a.candidates + n * kCounterStep, a.chunk_max = (float*)(a.mask + n * chunks * kMaskWords);
    a.row_max = a.chunk_max + n * chunks;
  }
  MDZ_WITH_ELEM(dtype, return launch_sample<E>(a, split, (hipStream_t)stream));
}

#pragma GCC visibility pop
}  // extern "C"
