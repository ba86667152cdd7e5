// Sampling: one token per row of logits from a given random number, with a temperature, top-k, top-p and min-p (include/medusa.h, "sampling").
//
// Mathematics.  A token's mass is exp((logit - largest) / temperature), held as a 64-bit integer in units of 2^-S of the largest's (S = 62 less the bits
// of the vocabulary's size, at most 50): integer sums do not depend on the order of atomics, and a row's masses always fit.  In the order of the logits
// (descending, ties to the lower index) everything that is asked of a row is a place in one running sum: top-k the mass of the first k, top-p the first
// token up to which p of that lies, min-p the mass of the logits from a border on; the kept tokens are the shortest of these beginnings, and the draw is the
// token at which the running sum passes u times their mass.  So nothing is sorted but the bin of a histogram in which such a place lies.
//
// Bins: 1024 steps of (largest - logit) / temperature, 1/32 each.  A place is found in the bins' running sums; of its bin the tokens are gathered and
// sorted, or, where they are more than kSortMost (ties, flat rows), cut again by their bits into 1024 until they are few or all equal.
#include "kernels.h"

namespace mdz {

constexpr int kBins = 1024;
constexpr float kBinsPerUnit = 32.f;
constexpr int kChunk = 4096;      // tokens of a workgroup where a row is split
constexpr int kSortMost = 2048;   // tokens of a bin that are sorted in LDS
constexpr int kMaskWords = kBins / 32;

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
  // split rows: per row and chunk the largest logit and which bins it has tokens in; per row the histogram
  float* chunk_max;
  uint32_t* mask;
  uint64_t* mass;
  uint32_t* count;
};

// a row's settings, and the largest of its logits
struct RowSettings {
  float inv_t, largest;
  double rate;  // log2(e) / temperature
  int top_k, shift;
  double top_p, min_p;
  __device__ inline RowSettings(const SampleArgs& a, int row, float max) {
    const int s = row / a.per;
    const float t = a.temperature ? a.temperature[s] : 1.f;
    const bool greedy = !(t > 0.f);
    largest = max, shift = a.shift;
    inv_t = greedy ? 1.f : fminf(1.f / t, 3.402823466e38f);
    rate = greedy ? 1.4426950408889634 : 1.4426950408889634 / (double)t;
    top_k = greedy ? 1 : a.top_k ? a.top_k[s] : 0;
    top_p = a.top_p ? (double)a.top_p[s] : 1.0;
    min_p = a.min_p ? (double)a.min_p[s] : 0.0;
  }
  // tokens that can be drawn: not NaN, not minus infinity; beside plus infinity nothing else
  __device__ inline bool valid(float l) const { return l > -INFINITY && (largest < INFINITY || l == largest); }
  // monotone in l: a difference, a product and a conversion of fp32
  __device__ inline int bin(float l) const {
    const float d = l == largest ? 0.f : fminf(largest - l, 3.402823466e38f) * inv_t;
    return (int)fminf(d * kBinsPerUnit, (float)(kBins - 1));
  }
  // 2^(shift + y), rounded to an integer; 2^f by its series, whose rest behind f^11 is below 7e-15 (the masses' steps are 2^-45 at 128000 tokens)
  __device__ inline uint64_t mass(float l) const {
    const double diff = l == largest ? 0.0 : (double)l - (double)largest;
    const double y = fmax(diff * rate, -1100.0), n = rint(y), f = y - n;
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
    // added to 2^52 a number is rounded to an integer, which the sum's mantissa is
    return __builtin_bit_cast(uint64_t, ldexp(e, (int)n + shift) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
  }
};

// logit i of a row (minus zero as zero: they tie)
template <typename T>
__device__ inline float logit(const T* row, int i) { return to_float(row[i]) + 0.f; }
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
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kChunk / 256; ++i) {
    const int at = first + i * 256 + (int)threadIdx.x;
    if (at < a.vocab) m = fmaxf(m, logit(l, at));
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

// The chunk's tokens into the row's histogram, through LDS, and which bins they are in.
template <typename T>
__global__ void __launch_bounds__(256) sample_bins_kernel(SampleArgs a) {
  __shared__ uint64_t mass[kBins];
  __shared__ uint32_t count[kBins];
  __shared__ float scratch[4];
  const int chunk = blockIdx.x, row = blockIdx.y, first = chunk * kChunk;
  const T* const l = reinterpret_cast<const T*>(a.logits) + row * a.ld;
  float v[kChunk / 256];
#pragma unroll
  for (int i = 0; i < kChunk / 256; ++i) {
    const int at = first + i * 256 + (int)threadIdx.x;
    v[i] = at < a.vocab ? logit(l, at) : -INFINITY;
  }
  for (int b = threadIdx.x; b < kBins; b += 256) mass[b] = 0, count[b] = 0;
  const RowSettings s(a, row, row_max<256>(a, row, scratch));
#pragma unroll
  for (int i = 0; i < kChunk / 256; ++i)
    if (s.valid(v[i])) {
      const int b = s.bin(v[i]);
      atomicAdd((unsigned long long*)&mass[b], (unsigned long long)s.mass(v[i]));
      atomicAdd(&count[b], 1u);
    }
  __syncthreads();
  for (int b = threadIdx.x; b < kBins; b += 256) {
    const uint32_t n = count[b];
    const uint64_t lanes = __ballot(n != 0);  // 64 bins: two words of the mask
    if ((threadIdx.x & 31) == 0) a.mask[((int64_t)row * a.chunks + chunk) * kMaskWords + (b >> 5)] = (uint32_t)(lanes >> (threadIdx.x & 32));
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

template <int NT>
struct RowLds {
  uint64_t mass[kBins];        // running sums of the row's histogram
  uint32_t count[kBins];
  union {
    struct {
      uint64_t list[kSortMost];  // ~key << 32 | index: sorted ascending these are the tokens in their order
      uint64_t through[kSortMost];
    };
    struct {
      uint64_t sub_mass[kBins];
      uint32_t sub_count[kBins];
    };
  };
  uint64_t scratch[2 * NT / 64];
  float fscratch[NT / 64];
  uint32_t uscratch[NT / 64];
  uint32_t n, found, listed;  // listed: the bin in `list`, or kBins
};

// calls f(logit, index) for the valid tokens of bin `b`
template <typename T, int NT, typename F>
__device__ inline void for_bin(const SampleArgs& a, const RowSettings& s, const T* l, int row, int b, F&& f) {
  for (int chunk = 0; chunk < a.chunks; ++chunk) {
    if (a.mask && !(a.mask[((int64_t)row * a.chunks + chunk) * kMaskWords + (b >> 5)] >> (b & 31) & 1u)) continue;
    const int end = min(a.vocab, (chunk + 1) * kChunk);
    for (int i = chunk * kChunk + (int)threadIdx.x; i < end; i += NT) {
      const float v = logit(l, i);
      if (s.valid(v) && s.bin(v) == b) f(v, i);
    }
  }
}

// the first of n running sums that reaches the target (the last, if none does); one thread finds it
template <int NT, typename Reached>
__device__ inline int first_reached(int n, uint32_t* found, Reached&& reached) {
  __syncthreads();
  if (threadIdx.x == 0) *found = n - 1;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += NT)
    if (reached(i) && (i == 0 || !reached(i - 1))) *found = i;
  __syncthreads();
  return (int)*found;
}

// Requires 1 <= target <= the row's count or mass.  (Loops and the list are bounded by themselves, whatever becomes of the logits meanwhile.)
template <typename T, int NT>
__device__ inline Place find_place(const SampleArgs& a, const RowSettings& s, const T* l, int row, RowLds<NT>& d, PlaceOf of, uint64_t target, bool want_index) {
  const int b = first_reached<NT>(kBins, &d.found, [&](int i) { return (of == PLACE_OF_COUNT ? (uint64_t)d.count[i] : d.mass[i]) >= target; });
  uint64_t before_mass = b ? d.mass[b - 1] : 0;
  uint32_t before_count = b ? d.count[b - 1] : 0, n = d.count[b] - before_count;
  uint32_t lo = 0, hi = 0xFFFFFFFFu;  // keys that are left of the bin
  for (int level = 0; n > kSortMost && level < 8; ++level) {
    __syncthreads();
    if (threadIdx.x == 0) d.listed = kBins;
    uint32_t least = 0xFFFFFFFFu, most = 0;
    for_bin<T, NT>(a, s, l, row, b, [&](float v, int) {
      const uint32_t k = order_key(v);
      if (k >= lo && k <= hi) least = min(least, k), most = max(most, k);
    });
    least = block_reduce<NT>(least, d.uscratch, [](uint32_t x, uint32_t y) { return min(x, y); });
    most = block_reduce<NT>(most, d.uscratch, [](uint32_t x, uint32_t y) { return max(x, y); });
    if (least >= most) {  // all equal: the place is a matter of counting
      const float v = __uint_as_float(most & 0x80000000u ? most & 0x7FFFFFFFu : ~most);
      const uint64_t w = s.mass(v);
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
    for (int i = threadIdx.x; i < kBins; i += NT) d.sub_mass[i] = 0, d.sub_count[i] = 0;
    __syncthreads();
    for_bin<T, NT>(a, s, l, row, b, [&](float v, int) {
      const uint32_t k = order_key(v);
      if (k < least || k > most) return;
      atomicAdd((unsigned long long*)&d.sub_mass[(most - k) >> shift], (unsigned long long)s.mass(v));
      atomicAdd(&d.sub_count[(most - k) >> shift], 1u);
    });
    running_sums<NT>(d.sub_mass, d.sub_count, d.scratch);
    const int c = first_reached<NT>(kBins, &d.found, [&](int i) {
      return (of == PLACE_OF_COUNT ? (uint64_t)before_count + d.sub_count[i] : before_mass + d.sub_mass[i]) >= target;
    });
    hi = most - ((uint32_t)c << shift);
    lo = max((uint64_t)least, (uint64_t)hi - min((uint64_t)hi, ((uint64_t)1 << shift) - 1));
    const uint64_t skipped = c ? d.sub_mass[c - 1] : 0;
    const uint32_t skipped_count = c ? d.sub_count[c - 1] : 0;
    n = d.sub_count[c] - skipped_count;
    before_mass += skipped, before_count += skipped_count;
    __syncthreads();
  }
  n = min(n, (uint32_t)kSortMost);
  const bool whole = lo == 0 && hi == 0xFFFFFFFFu;
  if (!whole || d.listed != (uint32_t)b) {
    int padded = 2;
    while (padded < (int)n) padded <<= 1;
    __syncthreads();
    if (threadIdx.x == 0) d.n = 0, d.listed = whole ? b : kBins;
    for (int i = (int)n + (int)threadIdx.x; i < padded; i += NT) d.list[i] = ~0ull;
    __syncthreads();
    for_bin<T, NT>(a, s, l, row, b, [&](float v, int i) {
      const uint32_t k = order_key(v);
      if (k < lo || k > hi) return;
      const uint32_t at = atomicAdd(&d.n, 1u);
      if (at < n) d.list[at] = (uint64_t)~k << 32 | (uint32_t)i;
    });
    for (int size = 2; size <= padded; size <<= 1)
      for (int step = size >> 1; step > 0; step >>= 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < padded / 2; i += NT) {
          const int x = 2 * i - (i & (step - 1)), y = x + step;
          const uint64_t u = d.list[x], v = d.list[y];
          if ((u > v) == !(x & size)) d.list[x] = v, d.list[y] = u;
        }
      }
    __syncthreads();
    // running masses: a wave at a time over 64 tokens (the first wave alone, the lists are short)
    if (threadIdx.x < 64) {
      uint64_t carry = 0;
      for (int first = 0; first < (int)n; first += 64) {
        const int i = first + (int)threadIdx.x;
        const uint32_t k = ~(uint32_t)(d.list[min(i, (int)n - 1)] >> 32);
        uint64_t m = i < (int)n ? s.mass(__uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k)) : 0;
#pragma unroll
        for (int e = 1; e < 64; e <<= 1) {
          const uint64_t o = __shfl_up((unsigned long long)m, e);
          if ((int)threadIdx.x >= e) m += o;
        }
        if (i < (int)n) d.through[i] = carry + m;
        carry += __shfl((unsigned long long)m, 63);
      }
    }
  }
  const int j = first_reached<NT>((int)n, &d.found, [&](int i) {
    return (of == PLACE_OF_COUNT ? (uint64_t)before_count + i + 1 : before_mass + d.through[i]) >= target;
  });
  return Place{before_mass + d.through[j], d.through[j] - (j ? d.through[j - 1] : 0), (int)(uint32_t)d.list[j]};
}

// d.mass and d.count: the row's histogram.  All threads; the first writes the row's answer.
template <typename T, int NT>
__device__ inline void draw_row(const SampleArgs& a, const RowSettings& s, const T* l, int row, RowLds<NT>& d) {
  if (threadIdx.x == 0) d.listed = kBins;
  running_sums<NT>(d.mass, d.count, d.scratch);
  const uint32_t n = d.count[kBins - 1];
  if (n == 0) {  // nothing to draw
    if (threadIdx.x == 0) {
      a.token[row] = -1;
      if (a.prob) a.prob[row] = 0.f;
    }
    return;
  }
  uint64_t kept = d.mass[kBins - 1];
  if (s.top_k > 0 && (uint32_t)s.top_k < n) kept = find_place<T, NT>(a, s, l, row, d, PLACE_OF_COUNT, (uint64_t)s.top_k, false).through;
  const uint64_t after_k = kept;
  if (s.top_p < 1.0) {
    const double p = ceil(fmax(s.top_p, 0.0) * (double)after_k);
    kept = find_place<T, NT>(a, s, l, row, d, PLACE_OF_MASS, min(max((uint64_t)p, (uint64_t)1), after_k), false).through;
  }
  if (s.min_p > 0.0 && s.largest < INFINITY && s.rate > 0.0) {  // (at an infinite temperature all masses are the largest)
    // mass >= min_p  <=>  logit >= largest + temperature ln(min_p)
    const double border = (double)s.largest + log2(fmin(s.min_p, 1.0)) / s.rate;
    const float edge = fmaxf((float)border, -3.402823466e38f);
    const int b = s.bin(fminf(edge, s.largest));
    // (the bins before that of the border's neighbours are whole; the border's rounding to fp32 may cross a bin)
    const int first = max(0, b - 1), last = min(kBins - 1, b + 1);
    uint64_t mass = 0;
    for (int i = first; i <= last; ++i)
      if (d.count[i] != (i ? d.count[i - 1] : 0))
        for_bin<T, NT>(a, s, l, row, i, [&](float v, int) {
          if ((double)v >= border) mass += s.mass(v);
        });
    mass = block_reduce<NT>((unsigned long long)mass, (unsigned long long*)d.scratch, [](unsigned long long x, unsigned long long y) { return x + y; });
    kept = min(kept, max((first ? d.mass[first - 1] : 0) + mass, (uint64_t)1 << s.shift));
  }
  const double u = (double)a.u[row], at = u > 0.0 ? u * (double)kept : 0.0;
  const uint64_t target = at < (double)(kept - 1) ? (uint64_t)at : kept - 1;
  const Place p = find_place<T, NT>(a, s, l, row, d, PLACE_OF_MASS, target + 1, true);
  if (threadIdx.x == 0) {
    a.token[row] = p.index;
    if (a.prob) a.prob[row] = (float)((double)p.mass / (double)kept);
  }
}

template <typename T>
__global__ void __launch_bounds__(512) sample_draw_kernel(SampleArgs a) {
  __shared__ RowLds<512> d;
  const int row = blockIdx.x;
  for (int b = threadIdx.x; b < kBins; b += 512) d.mass[b] = a.mass[(int64_t)row * kBins + b], d.count[b] = a.count[(int64_t)row * kBins + b];
  const RowSettings s(a, row, row_max<512>(a, row, d.fscratch));
  draw_row<T, 512>(a, s, reinterpret_cast<const T*>(a.logits) + row * a.ld, row, d);
}

// A row to a workgroup: all passes.
template <typename T>
__global__ void __launch_bounds__(1024) sample_row_kernel(SampleArgs a) {
  __shared__ RowLds<1024> d;
  const int row = blockIdx.x;
  const T* const l = reinterpret_cast<const T*>(a.logits) + row * a.ld;
  float m = -INFINITY;
  for (int i = threadIdx.x; i < a.vocab; i += 1024) m = fmaxf(m, logit(l, i));
  for (int b = threadIdx.x; b < kBins; b += 1024) d.mass[b] = 0, d.count[b] = 0;
  const RowSettings s(a, row, block_reduce<1024>(m, d.fscratch, [](float x, float y) { return fmaxf(x, y); }));
  for (int i = threadIdx.x; i < a.vocab; i += 1024) {
    const float v = logit(l, i);
    if (s.valid(v)) {
      const int b = s.bin(v);
      atomicAdd((unsigned long long*)&d.mass[b], (unsigned long long)s.mass(v));
      atomicAdd(&d.count[b], 1u);
    }
  }
  draw_row<T, 1024>(a, s, l, row, d);
}

// ---- the call ----------------------------------------------------------------------------------------------
constexpr int kMaxVocab = 1 << 24;  // the masses then still have 38 bits behind the point
static bool sample_splits(int rows, int vocab) { return vocab > 2 * kChunk && rows < num_cus(); }
static int64_t sample_bytes(int rows, int vocab) {
  if (!sample_splits(rows, vocab)) return 0;
  const int64_t chunks = (vocab + kChunk - 1) / kChunk;
  return rows * (kBins * 12 + chunks * (kMaskWords * 4 + 4));
}
static int check_sample(int rows, int vocab) {
  MDZ_REQUIRE(rows >= 0 && vocab > 0, MDZ_EINVAL, "sample: %d rows of %d logits", rows, vocab);
  MDZ_REQUIRE(vocab <= kMaxVocab && rows <= 1 << 21, MDZ_EUNSUPPORTED, "sample: up to 2^21 rows of 2^24 logits (%d of %d)", rows, vocab);
  return MDZ_OK;
}

template <typename T>
static int launch_sample(const SampleArgs& a, bool split, hipStream_t st) {
  if (!split) {
    launch_timed(PROF_SELECT, sample_row_kernel<T>, (unsigned)a.rows, 1024, 0, st, a);
    MDZ_LAUNCH_CHECK();
    return MDZ_OK;
  }
  launch_timed(PROF_SELECT, sample_max_kernel<T>, dim3(a.chunks, a.rows), 256, 0, st, a);
  MDZ_LAUNCH_CHECK();
  launch_timed(PROF_SELECT, sample_bins_kernel<T>, dim3(a.chunks, a.rows), 256, 0, st, a);
  MDZ_LAUNCH_CHECK();
  launch_timed(PROF_SELECT, sample_draw_kernel<T>, (unsigned)a.rows, 512, 0, st, a);
  MDZ_LAUNCH_CHECK();
  return MDZ_OK;
}

}  // namespace mdz

using namespace mdz;

extern "C" {
#pragma GCC visibility push(default)

int64_t medusa_sample_workspace_bytes(int rows, int vocab) {
  const int rc = check_sample(rows, vocab);
  return rc ? rc : sample_bytes(rows, vocab);
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
    a.mass = (uint64_t*)ws;
    a.count = (uint32_t*)(a.mass + (int64_t)rows * kBins);
    a.mask = a.count + (int64_t)rows * kBins;
    a.chunk_max = (float*)(a.mask + (int64_t)rows * a.chunks * kMaskWords);
  }
  MDZ_WITH_ELEM(dtype, return launch_sample<E>(a, split, (hipStream_t)stream));
}

#pragma GCC visibility pop
}  // extern "C"
