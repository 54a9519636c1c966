// A word for every row of logits.  e = exp((x - top) / temperature); the words in the order of their logits (equal ones by number) are cut off behind the first top_k, where less than
// top_p of the sum of those lies in front, and at e = min_p: all three leave the first so many of one order.  So the row is not sorted: a histogram of it over eighths of a power of two of e
// says in which step of it a cut lies.  If the words up to there are at most one to a thread of a workgroup, those are sorted and the rest is not looked at again; else only the words of
// that step are.
//
// One row of 32000 words with all three cuts takes 3.2 + 6.8 + 10.8 us (tops, histograms, choice), 64 rows of 128256 in bf16 with every kind of cut 5.7 + 11.3 + 53.5.  The choice is one workgroup's
// work and bound by what that can do: a walk over a row of 128256 words takes it 7 us and more with much to do on the way, so the shorter way (32 us for the one row without it) and what is kept in
// LDS count (the 64 rows: 71 where the words of a step were sorted 2048 at a time and looked for in the row again).  Up to 512 words are sorted by counting each one's place (64: 4 us less than in
// steps).  Steps of a 32nd do not help: the many words of a flat row are far below its top.
//
// Answers are whole numbers, so sums are kept in 64 bits and in whole numbers where workgroups' order could show: a word of step b counts 1 and the
// 2^-40ths by which e 2^(b / 8) is below 1, both in one 64-bit addition in LDS.  Rounding that to 2^-41 moves a sum by less than 1e-12 of itself, and the sum of words as large as the largest, of which there
// may be nothing else, not at all: each counts 1.
#pragma once
#include "verify_kernels.hpp"

namespace dpllm {

constexpr int kSampleBins = 512;            // e down to 2^-64
constexpr int kSampleThreads = 1024;        // of the workgroup that chooses
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kSampleList = 2048;           // words that LDS holds
constexpr int kSampleSort = 512;            // and that are sorted, but for those of the shorter way
constexpr int kSampleChunks = 1088;         // at most, of a row of 2^22 words
constexpr int kPast = 1 << 12;              // more than a list is long
constexpr int kCountShift = 50;             // a chunk has at most 2^13 words of less than 2^37 each

struct SampleTop {      // of a chunk: its largest logit and where that is first
  float top;
  int at;
};

struct SampleArgs {
  const char* logits;
  int64_t stride;               // elements
  const float *uniforms, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t *words, *kept;
  SampleTop* tops;              // [rows][chunks]
  unsigned long long* bins;     // [rows][chunks][kSampleBins]
  int rows, vocabulary, chunks;
};

// Where a word lies.  y = 2^19 - t, t the 256ths of a power of two by which e is below 1, so that the upper word of y has all whole numbers in it and its last bits count 2^-34: an error of 8e-14 of
// e.  Step b is t in (32 b, 32 (b + 1)], the first with 0; r = y - floor(y) is what is left to the next whole t, and with the five bits of y above that to the step's end: e is the step's first e, 2^(-b / 8), times
// 2^((bits - 32) / 256) 2^(r / 256).  1 + c1 r + c2 r^2 + c3 r^3 is the last of these to 2e-14.  A dozen instructions in 64 bits; with the series of the whole exponent they were 30,
// and the histograms of 64 rows of 128256 words took 14 us, now 11.
constexpr int kSampleTable = 32;      // 2^40 2^((j - 32) / 256)
struct Steps {
  float top;
  double steps;      // 256 / (temperature ln 2)
  const double* table;
  __device__ __forceinline__ Steps(float top, float temperature, const double* table) : top(top), steps(369.32993046757462 / (double)temperature), table(table) {}
  __device__ __forceinline__ double place(float x) const {
    const double t = x == top ? 0.0 : ((double)x - (double)top) * steps;
    return __builtin_fmin(__builtin_fmax(t, -131072.0) + 524288.0, 524288.0 - 0x1p-34);      // (NaN counts as far below)
  }
  // Its step; kSampleBins or more: it is left out (as are NaN and minus infinity).
  __device__ __forceinline__ static int bin(double y) { return (int)((~(uint32_t)(__builtin_bit_cast(uint64_t, y) >> 32) & 0xfffffu) >> 7); }
  // e by the first of its step, times 2^40 w, plus c
  __device__ __forceinline__ double share(double y, double w, double c) const {
    const double r = __builtin_amdgcn_fract(y);
    double f = __builtin_fma(r, 3.312607527945956e-09, 3.6655631008313955e-06);
    f = __builtin_fma(f, r, 0.0027076061744736664);
    f = __builtin_fma(f, r, 1.0);
    return __builtin_fma(f, table[(uint32_t)(__builtin_bit_cast(uint64_t, y) >> 34) & (kSampleTable - 1)] * w, c);
  }
  // What that is below 1, in 2^-40ths, to the nearest; that of the largest logit, whose y is 2^-34 short of 2^19, is 0.
  __device__ __forceinline__ unsigned long long lack(double y) const {
    return __builtin_bit_cast(uint64_t, share(y, -1.0, 0x1p52 + 0x1p40)) & ((1ull << 52) - 1);
  }
};
// Fills the table; a barrier has to follow.
__device__ __forceinline__ void fill_steps(double* table) {
  if (threadIdx.x < kSampleTable) table[threadIdx.x] = 0x1p40 * exp_of(((int)threadIdx.x - kSampleTable) * 0.0027076061740622863);      // ln 2 / 256
}
__device__ __forceinline__ double base_of(int bin) { return exp_of(-0.086643397569993164 * bin); }      // the first e of a step, which none of its is above: ln 2 / 8
__device__ __forceinline__ float larger(float x, float y) { return fmaxf(x, y); }
__device__ __forceinline__ int smaller(int x, int y) { return min(x, y); }

// A piece of a row from word i on (16-byte aligned, perhaps in front of the row's first or past its last); what lies outside is NaN.
template <typename T>
__device__ __forceinline__ typename Piece<T>::type piece_at(const char* row, int n, int i) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  constexpr int E = Piece<T>::E, EACH = 4 / sizeof(T);      // words to 32 bits
  const T* words = reinterpret_cast<const T*>(row);
  if (i >= 0 && i + E <= n) return *reinterpret_cast<const typename Piece<T>::type*>(words + i);
  u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll 1
  for (int e = 0; e < E; ++e) {
    const T x = i + e >= 0 && i + e < n ? words[i + e] : (T)__builtin_nanf("");
    uint32_t w;
    if constexpr (sizeof(T) == 4)
      w = __builtin_bit_cast(uint32_t, x);
    else
      w = (uint32_t)__builtin_bit_cast(uint16_t, x) << 16 * (e % EACH);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] |= e / EACH == j ? w : 0u;
  }
  return __builtin_bit_cast(typename Piece<T>::type, v);
}

// f(piece, its first word) for the pieces of a stretch of a row that a group of `threads` threads shares, four on their way at a time, those of a thread in their order.
template <typename T, typename F>
__device__ __forceinline__ void each_piece(const char* row, int n, int first, int pieces, int thread, int threads, F f) {
  constexpr int E = Piece<T>::E;
  for (int p0 = thread; p0 < pieces; p0 += 4 * threads) {
    typename Piece<T>::type v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = piece_at<T>(row, n, first + (p0 + j * threads < pieces ? p0 + j * threads : p0) * E);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (p0 + j * threads < pieces) f(v[j], first + (p0 + j * threads) * E);
  }
}

// f(x, i) for those of a piece that are within [low, high].  They are few, or dear: so f's code is there once.
template <typename T, typename F>
__device__ __forceinline__ void each_between(const typename Piece<T>::type& v, int first, float low, float high, F f) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 w = __builtin_bit_cast(u32x4, v);
  uint32_t in = 0;
#pragma unroll
  for (int e = 0; e < Piece<T>::E; ++e) in |= (float)v[e] >= low && (float)v[e] <= high ? 1u << e : 0u;
#pragma unroll 1
  while (in != 0) {
    const int e = __builtin_ctz(in), d = e * (int)sizeof(T) / 4;
    const uint32_t here = d < 2 ? (d == 0 ? w[0] : w[1]) : (d == 2 ? w[2] : w[3]);
    if constexpr (sizeof(T) == 4)
      f(__uint_as_float(here), first + e);
    else
      f((float)__builtin_bit_cast(T, (uint16_t)(e & 1 ? here >> 16 : here)), first + e);
    in &= in - 1;
  }
}

// Workgroups of a row's chunks: x is the row, so that with eight rows or more (their number rounded up to a multiple) all of them and the one that chooses are on the same die
// and find the row in its cache.
// The largest logit of a chunk.
template <typename T>
__global__ void __launch_bounds__(kVerThreads) sample_tops_kernel(const SampleArgs a) {
  __shared__ float tops[kVerThreads / 64];
  __shared__ int places[kVerThreads / 64];
  const int row = blockIdx.x, chunk = blockIdx.y;
  if (row >= a.rows) return;
  const char* from = a.logits + row * a.stride * (int64_t)sizeof(T);
  float mine = -INFINITY;
  int at = 0x7fffffff;
  each_piece<T>(from, a.vocabulary, chunk * Chunk<T>::kElements - Chunk<T>::lead(from), Chunk<T>::kElements / Chunk<T>::E, threadIdx.x, kVerThreads,
                [&](const typename Piece<T>::type& v, int i) {
#pragma unroll
                  for (int e = 0; e < Chunk<T>::E; ++e)
                    if ((float)v[e] > mine) {
                      mine = (float)v[e];
                      at = i + e;
                    }
                });
  const float top = wave_all(mine, larger);
  if (mine != top) at = 0x7fffffff;
  at = wave_all(at, smaller);
  if ((threadIdx.x & 63) == 0) {
    tops[threadIdx.x >> 6] = top;
    places[threadIdx.x >> 6] = at;
  }
  __syncthreads();
  if (threadIdx.x > 0) return;
  SampleTop best{tops[0], places[0]};
  for (int w = 1; w < kVerThreads / 64; ++w)
    if (tops[w] > best.top || (tops[w] == best.top && places[w] < best.at)) best = {tops[w], places[w]};
  a.tops[(int64_t)row * a.chunks + chunk] = best;
}

// The histogram of a chunk.
template <typename T>
__global__ void __launch_bounds__(kVerThreads) sample_bins_kernel(const SampleArgs a) {
  __shared__ unsigned long long bins[kSampleBins];
  __shared__ double table[kSampleTable];
  const int row = blockIdx.x, chunk = blockIdx.y;
  if (row >= a.rows) return;
  const float temperature = a.temperature[row];
  if (greedy(temperature)) return;
  const char* from = a.logits + row * a.stride * (int64_t)sizeof(T);
  for (int i = threadIdx.x; i < kSampleBins; i += kVerThreads) bins[i] = 0;
  fill_steps(table);
  float top = -INFINITY;
  for (int i = threadIdx.x & 63; i < a.chunks; i += 64) top = fmaxf(top, a.tops[(int64_t)row * a.chunks + i].top);
  top = wave_all(top, larger);
  __syncthreads();
  if (top == -INFINITY) return;
  const Steps steps(top, temperature, table);
  each_piece<T>(from, a.vocabulary, chunk * Chunk<T>::kElements - Chunk<T>::lead(from), Chunk<T>::kElements / Chunk<T>::E, threadIdx.x, kVerThreads,
                [&](const typename Piece<T>::type& v, int) {
#pragma unroll
                  for (int e = 0; e < Chunk<T>::E; ++e) {
                    const double y = steps.place((float)v[e]);
                    if (steps.bin(y) < kSampleBins) atomicAdd(&bins[steps.bin(y)], (1ull << kCountShift) + steps.lack(y));
                  }
                });
  __syncthreads();
  for (int i = threadIdx.x; i < kSampleBins; i += kVerThreads) a.bins[((int64_t)row * a.chunks + chunk) * kSampleBins + i] = bins[i];
}

// Words in front of a cut: those above its logit, and of those at it the ones up to a number.
struct Cut {
  float at;
  int upto;
  __device__ __forceinline__ bool has(float x, int i) const { return x > at || (x == at && i <= upto); }
};

// Floats as whole numbers in the same order (-0 and 0 are one); of narrower types without the bits that all of theirs share.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t w = __float_as_uint(x + 0.f);
  return w >> 31 ? ~w : w | 0x80000000u;
}
__device__ __forceinline__ float from_key(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }
template <typename T>
struct Narrow {
  static constexpr int kShared = std::is_same<T, float>::value ? 0 : std::is_same<T, half_t>::value ? 13 : 16;
  __device__ __forceinline__ static uint32_t of(float x) { return key_of(x) >> kShared; }
  __device__ __forceinline__ static float back(uint32_t k) {
    const uint32_t w = k << kShared;
    return from_key(w >> 31 ? w : w | ((1u << kShared) - 1u));
  }
};

struct SampleSpace {
  unsigned long long list[kSampleList];     // ~key << 32 | number
  unsigned long long chunks[kSampleChunks];
  double base[kSampleBins];                 // the first e of a bin, in 2^-40ths
  double table[kSampleTable];
  double sums[kSampleBins];                 // running, over bins
  uint32_t counts[kSampleBins];
  unsigned long long fine[kSampleBins];     // of a step that is looked at more closely
  uint32_t fine_counts[kSampleBins];
  double wave_sums[kSampleWaves];
  uint32_t wave_counts[kSampleWaves];
  double sum, sum_before;
  int found, before, length;
  int listed, listed_bin;                   // the list has all words of a bin: how many (else 0), and which
};

// The sum of what the first `waves` wavefronts left in s.wave_sums.
__device__ __forceinline__ double of_waves(const SampleSpace& s, int waves) {
  const int lane = threadIdx.x & 63;
  return wave_sum(lane < waves ? s.wave_sums[lane & (kSampleWaves - 1)] : 0.0);
}

// The running sums of kSampleBins values and counts, one of each to a thread of the first eight wavefronts, into s.sums and s.counts.
__device__ __forceinline__ void run_bins(SampleSpace& s, double sum, uint32_t count) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const double upto = wave_scan(sum), number = wave_scan((double)count);      // (whole numbers)
  __syncthreads();
  if (lane == 63) {
    s.wave_sums[wave] = upto;
    s.wave_counts[wave] = (uint32_t)number;
  }
  __syncthreads();
  const double plus = of_waves(s, wave), more = wave_sum(lane < wave ? (double)s.wave_counts[lane & (kSampleWaves - 1)] : 0.0);
  if (threadIdx.x < kSampleBins) {
    s.sums[threadIdx.x] = upto + plus;
    s.counts[threadIdx.x] = (uint32_t)(number + more);
  }
  __syncthreads();
}

// The first bin with words up to which there are `count` words, or (count 0) a sum of `sum`; the last one with words if there is none.  s.found, s.before and s.sum_before: what lies in front.
// A running sum is added up in another order for each bin, so next to one it may be less, or exceed it without a word in between, by their rounding: bins without words are passed over, and the lowest that fits
// is the one.
__device__ __forceinline__ void find_bin(SampleSpace& s, uint32_t count, double sum) {
  const int b = threadIdx.x;
  uint32_t front = 0;
  if (b < kSampleBins) {
    const uint32_t upto = s.counts[b], all = s.counts[kSampleBins - 1];
    front = b == 0 ? 0u : s.counts[b - 1];
    const uint64_t fits = __ballot(upto > front && (upto == all || (count > 0 ? upto >= count : s.sums[b] >= sum)));
    if ((b & 63) == 0) s.wave_counts[b >> 6] = fits == 0 ? kSampleBins - 1 : b + __builtin_ctzll(fits);
  }
  __syncthreads();
  uint32_t first = kSampleBins - 1;
#pragma unroll
  for (int w = 0; w < kSampleBins / 64; ++w) first = min(first, s.wave_counts[w]);
  if (b == (int)first) {
    s.found = b;
    s.before = (int)front;
    s.sum_before = b == 0 ? 0.0 : s.sums[b - 1];
  }
  __syncthreads();
}

// f(x, i) for all words of a row whose logits are within [low, high], in no order.
template <typename T, typename F>
__device__ __forceinline__ void words_between(const char* row, int n, float low, float high, F f) {
  constexpr int E = Piece<T>::E;
  const int lead = Chunk<T>::lead(row);
  each_piece<T>(row, n, -lead, (n + lead + E - 1) / E, threadIdx.x, kSampleThreads,
                [&](const typename Piece<T>::type& v, int i) { each_between<T>(v, i, low, high, f); });
}

// Sorts n (a power of two) different numbers, or such that are all ones, the smallest first.  Up to 512: each is put where as many are smaller; the whole workgroup counts.  `space`: as many more.
// More: in steps, those whose partners are at most 64 apart in the 128 numbers of a wavefront.
__device__ __forceinline__ void sort(unsigned long long* list, int n, uint32_t* ranks, unsigned long long* space) {
  if (n <= 512) {
    const int i = threadIdx.x & (n - 1), parts = kSampleThreads / n, each = (n + parts - 1) / parts, begin = (int)threadIdx.x / n * each;
    if ((int)threadIdx.x < n) ranks[threadIdx.x] = 0;
    __syncthreads();
    const unsigned long long mine = list[i];
    uint32_t rank = 0;
#pragma unroll 8
    for (int j = begin; j < begin + each; ++j) rank += j < n && (list[j] < mine || (list[j] == mine && j < i));
    atomicAdd(&ranks[i], rank);
    __syncthreads();
    if ((int)threadIdx.x < n) space[ranks[i]] = mine;
    __syncthreads();
    if ((int)threadIdx.x < n) list[i] = space[i];
    __syncthreads();
    return;
  }
#pragma unroll 1
  for (int size = 2; size <= n; size *= 2)
#pragma unroll 1
    for (int gap = size / 2; gap > 0; gap /= 2) {
      for (int i = threadIdx.x; i < n / 2; i += kSampleThreads) {
        const int p = 2 * i - (i & (gap - 1)), q = p + gap;
        const unsigned long long x = list[p], y = list[q];
        if ((x > y) == ((p & size) == 0)) {
          list[p] = y;
          list[q] = x;
        }
      }
      const int next = gap > 1 ? gap / 2 : size;      // the next step's
      if (gap > 64 || next > 64) {
        __syncthreads();
      } else {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
    }
  __syncthreads();
}

// The running sum over the workgroup of a value of each thread.
__device__ __forceinline__ double group_scan(SampleSpace& s, double v) {
  const int wave = threadIdx.x >> 6;
  double upto = wave_scan(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) s.wave_sums[wave] = upto;
  __syncthreads();
  return upto + of_waves(s, wave);
}

// The order of the row as its histogram's bins are; all threads take part in each of these.
template <typename T>
struct Sampler {
  const SampleArgs& a;
  SampleSpace& s;
  int a_row;
  const char* row;
  float top;
  double by;      // eighths of a power of two
  const Steps& steps;

  __device__ __forceinline__ double e_at(double y) const { return steps.share(y, s.base[min(steps.bin(y), kSampleBins - 1)], 0.0); }
  __device__ __forceinline__ double e_of(float x) const { return x == top ? 1.0 : e_at(steps.place(x)); }
  // Bounds of the logits of bins first ... last, a little wide: by the rounding to a float, and by much more than places are rounded by.
  __device__ __forceinline__ float wide(float x) const { return __builtin_fabsf(x) * 0x1p-20f + (float)(0x1p-25 / by) + 0x1p-120f; }
  __device__ __forceinline__ float lowest(int last) const {
    if (top == INFINITY) return top;
    const float x = (float)((double)top - (last + 1) / by), low = x - wide(x);
    return low != low || last >= kSampleBins - 1 ? -INFINITY : low;
  }
  __device__ __forceinline__ float highest(int first) const {
    const float x = (float)((double)top - first / by), high = x + wide(x);
    return first == 0 || high != high ? INFINITY : high;
  }
  __device__ __forceinline__ float listed_logit(int i) const { return from_key(~(uint32_t)(s.list[i] >> 32)); }
  // The words of bin `bin` in front of a cut: `count` of them, or (count 0) those in front of which less than `sum` of them lies, at least one.  s.length and s.sum: how many, and their sum.
  __device__ Cut cut_in(int bin, int words, uint32_t count, double sum) {
    typedef Narrow<T> Key;
    uint32_t low = Key::of(lowest(bin)), high = Key::of(fminf(highest(bin), top));
    const double base = s.base[bin];
    int taken = 0;
    double taken_sum = 0.0;
    const auto inside = [&](float x, double y) {
      const uint32_t k = Key::of(x);
      return k >= low && k <= high && steps.bin(y) == bin;
    };
    int listed = 0;
    // narrower, until the words can be sorted or are all the same: nine of the key's 32 bits at a time, over the row until LDS holds the words, then over those
    for (int round = 0;; ++round) {
      if (listed == 0 && words <= kSampleList) {
        listed = words;
        if (threadIdx.x == 0) {
          s.length = 0;
          s.listed = round == 0 ? words : 0;
          s.listed_bin = bin;
        }
        __syncthreads();
        words_between<T>(row, a.vocabulary, Key::back(low), Key::back(high), [&](float x, int i) {
          if (inside(x, steps.place(x))) {
            const int at = atomicAdd(&s.length, 1);
            if (at < kSampleList) s.list[at] = (unsigned long long)~key_of(x) << 32 | (uint32_t)i;
          }
        });
        __syncthreads();
      }
      if (words <= kSampleSort || low == high || round == 4) break;
      if (threadIdx.x < kSampleBins) {
        s.fine[threadIdx.x] = 0;
        s.fine_counts[threadIdx.x] = 0;
      }
      __syncthreads();
      const int shift = max(0, 23 - __builtin_clz(high - low));      // (high - low) >> shift is below 512
      const auto add = [&](float x) {
        const double y = steps.place(x);
        if (inside(x, y)) {
          atomicAdd(&s.fine_counts[(high - Key::of(x)) >> shift], 1u);
          atomicAdd(&s.fine[(high - Key::of(x)) >> shift], steps.lack(y));
        }
      };
      if (listed > 0)
        for (int i = threadIdx.x; i < listed; i += kSampleThreads) add(listed_logit(i));
      else
        words_between<T>(row, a.vocabulary, Key::back(low), Key::back(high), [&](float x, int) { add(x); });
      __syncthreads();
      const int i = min((int)threadIdx.x, kSampleBins - 1);
      run_bins(s, base * ((double)s.fine_counts[i] * 0x1p40 - (double)s.fine[i]), s.fine_counts[i]);
      find_bin(s, count > 0 ? count - taken : 0u, sum - taken_sum);
      taken += s.before;
      taken_sum += s.sum_before;
      words = (int)(s.counts[s.found] - s.before);
      const uint32_t upper = high - ((uint32_t)s.found << shift), width = (1u << shift) - 1u;
      low = max(low, upper - min(upper, width));
      high = upper;
      __syncthreads();
    }
    if (words <= kSampleSort) {
      unsigned long long* few = s.fine;
      int size = 2;
      while (size < words) size *= 2;
      if (threadIdx.x == 0) s.length = 0;
      if ((int)threadIdx.x < size) few[threadIdx.x] = ~0ull;
      __syncthreads();
      for (int i = threadIdx.x; i < listed; i += kSampleThreads) {
        const float x = listed_logit(i);
        if (inside(x, steps.place(x))) few[atomicAdd(&s.length, 1) & (kSampleSort - 1)] = s.list[i];
      }
      __syncthreads();
      sort(few, size, s.fine_counts, reinterpret_cast<unsigned long long*>(s.sums));
      const int i = threadIdx.x;
      const double e = i < words ? e_of(from_key(~(uint32_t)(few[i] >> 32))) : 0.0, upto = group_scan(s, e), front = upto - e;
      if (i == 0) s.found = -1;
      __syncthreads();
      const bool stays = i < words && (count > 0 ? (uint32_t)(taken + i) < count : i + taken == 0 || taken_sum + front < sum);
      if (stays) atomicMax(&s.found, i);
      __syncthreads();
      if (stays && i == s.found) s.sum = taken_sum + upto;
      const int found = max(s.found, 0);
      if (i == 0) {
        s.length = taken + s.found + 1;
        if (s.found < 0) s.sum = taken_sum;
      }
      const unsigned long long w = few[found];
      __syncthreads();
      // (rounding between two ways to the same sum may leave none of these, as what is left of it may come to nothing or less: then the cut is in front of the first)
      if (s.length == taken) return {from_key(~(uint32_t)(w >> 32)), -1};
      return {from_key(~(uint32_t)(w >> 32)), (int)(uint32_t)w};
    }
    // all the same: so many of them by their numbers
    const float x = Key::back(high);
    const double e = e_of(x);
    int n = count > 0 ? (int)count - taken : (int)fmin((sum - taken_sum) / e, (double)words);
    if (count == 0) {
      while (n > 0 && (n - 1) * e >= sum - taken_sum) --n;
      while (n < words && n * e < sum - taken_sum) ++n;
    }
    n = min(max(n, 1), words);
    int upto = 0x7fffffff;
    if (n < words) {
      // the n-th by number: first in which chunk, then there
      typedef Chunk<T> C;
      uint32_t* in_chunk = reinterpret_cast<uint32_t*>(s.chunks);
      for (int c = threadIdx.x >> 6; c < a.chunks; c += kSampleWaves) {
        int mine = 0;
        each_piece<T>(row, a.vocabulary, c * C::kElements - C::lead(row), C::kElements / C::E, threadIdx.x & 63, 64, [&](const typename Piece<T>::type& v, int) {
#pragma unroll
          for (int j = 0; j < C::E; ++j) mine += (float)v[j] == x;
        });
        mine = (int)wave_sum((double)mine);
        if ((threadIdx.x & 63) == 0) in_chunk[c] = (uint32_t)mine;
      }
      __syncthreads();
      int two[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) two[j] = 2 * (int)threadIdx.x + j < a.chunks ? (int)in_chunk[2 * threadIdx.x + j] : 0;
      int before = (int)group_scan(s, (double)(two[0] + two[1])) - two[0] - two[1];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (before < n && n <= before + two[j]) {
          s.found = 2 * (int)threadIdx.x + j;
          s.before = before;
        }
        before += two[j];
      }
      __syncthreads();
      constexpr int EACH = C::kElements / kSampleThreads;
      const int first = s.found * C::kElements + EACH * (int)threadIdx.x - C::lead(row), wanted = n - s.before;
      static_assert(EACH == C::E, "a piece to a thread");
      const typename Piece<T>::type v = piece_at<T>(row, a.vocabulary, first);
      int mine = 0;
#pragma unroll
      for (int j = 0; j < EACH; ++j) mine += (float)v[j] == x;
      int k = (int)group_scan(s, (double)mine) - mine;
      if (k < wanted && wanted <= k + mine)
#pragma unroll
        for (int j = 0; j < EACH; ++j)
          if ((float)v[j] == x && ++k == wanted) s.found = first + j;
      __syncthreads();
      upto = s.found;
    }
    if (threadIdx.x == 0) {
      s.length = taken + n;
      s.sum = taken_sum + n * e;
    }
    __syncthreads();
    return {x, upto};
  }

  // The draw among the `words` words (at most one to a thread) of bins up to `bound`: the first k of them, of those the first up to p of `whole` (below 0: of their sum), of those with e of `least` or more.
  __device__ void draw(int bound, int words, int k, double whole, double p, double least) {
    if (threadIdx.x == 0) {
      s.length = 0;
      s.found = 0;
      s.before = 0x7fffffff;
    }
    int size = 2;
    while (size < words) size *= 2;
    if ((int)threadIdx.x < size) s.list[threadIdx.x] = ~0ull;
    __syncthreads();
    words_between<T>(row, a.vocabulary, lowest(bound), INFINITY, [&](float x, int i) {
      if (steps.bin(steps.place(x)) <= bound) s.list[atomicAdd(&s.length, 1) & (kSampleThreads - 1)] = (unsigned long long)~key_of(x) << 32 | (uint32_t)i;
    });
    __syncthreads();
    sort(s.list, size, s.fine_counts, s.fine);
    const int i = threadIdx.x, word = (int)(uint32_t)s.list[i];
    const double e = i < words ? e_of(from_key(~(uint32_t)(s.list[i] >> 32))) : 0.0;
    double upto = group_scan(s, e);
    if (i == min(k, words) - 1) s.sum = upto;
    __syncthreads();
    const double part = whole < 0.0 ? s.sum : whole;
    const bool stays = i < words && i < k && (i == 0 || ((p >= 1.0 || upto - e < p * part) && (least == 0.0 || e >= least)));
    const uint64_t these = __ballot(stays);
    if (these != 0 && (threadIdx.x & 63) == 0) atomicMax(&s.found, (int)threadIdx.x + 64 - __builtin_clzll(these));
    __syncthreads();
    const int kept = s.found;
    if (i == kept - 1) s.sum_before = upto;
    double* weights = reinterpret_cast<double*>(s.list + kSampleThreads);
    weights[i] = e;
    __syncthreads();
    const double want = (double)a.uniforms[a_row] * s.sum_before;
    // in the order of the words' numbers: of a few, eight lanes add up all in front of each; more are sorted again
    if (kept <= kSampleThreads / 8) {
      const int t = i / 8, number = (int)(uint32_t)s.list[t];
      double run = 0.0;
#pragma unroll 4
      for (int j = i & 7; j < kept; j += 8) run += (int)(uint32_t)s.list[j] <= number ? weights[j] : 0.0;
      run = team_all(run, 8, [](double x, double y) { return x + y; });
      if (t < kept && (i & 7) == 0) {
        atomicMax(&s.length, number + kPast);
        if (run > want) atomicMin(&s.before, number);
      }
    } else {
      s.list[i] = i < kept ? (unsigned long long)(uint32_t)word << 32 | (uint32_t)i : ~0ull;
      __syncthreads();
      sort(s.list, size, s.fine_counts, s.fine);
      const int number = (int)(uint32_t)(s.list[i] >> 32);
      const double run = group_scan(s, i < kept ? weights[(uint32_t)s.list[i]] : 0.0);
      if (i == kept - 1) atomicMax(&s.length, number + kPast);
      if (i < kept && run > want) atomicMin(&s.before, number);
    }
    __syncthreads();
    if (i == 0) {
      a.words[a_row] = min(s.before, s.length - kPast);      // (rounding may leave the sum short of its whole: then it is the last that stays)
      if (a.kept != nullptr) a.kept[a_row] = kept;
    }
  }
};

// One workgroup to a row.
template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_choose_kernel(const SampleArgs a) {
  __shared__ SampleSpace s;
  const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float temperature = a.temperature[row];
  const char* from = a.logits + row * a.stride * (int64_t)sizeof(T);
  const SampleTop* tops = a.tops + (int64_t)row * a.chunks;
  float top = -INFINITY;
  for (int i = lane; i < a.chunks; i += 64) top = fmaxf(top, tops[i].top);
  top = wave_all(top, larger);
  if (greedy(temperature) || top == -INFINITY) {
    int at = 0x7fffffff;
    for (int i = lane; i < a.chunks; i += 64) at = tops[i].top == top ? min(at, tops[i].at) : at;
    at = wave_all(at, smaller);
    if (threadIdx.x == 0) {
      a.words[row] = top == -INFINITY ? -1 : at;
      if (a.kept != nullptr) a.kept[row] = top == -INFINITY ? 0 : 1;
    }
    return;
  }
  const unsigned long long* bins = a.bins + (int64_t)row * a.chunks * kSampleBins;
  constexpr unsigned long long kMask = (1ull << kCountShift) - 1;

  // the bins of the row: two threads to each
  {
    fill_steps(s.table);
    const int b = threadIdx.x & (kSampleBins - 1), half = threadIdx.x / kSampleBins;
    uint32_t count = 0;
    unsigned long long less = 0;
#pragma unroll 4
    for (int c = half; c < a.chunks; c += 2) {
      const unsigned long long w = bins[(int64_t)c * kSampleBins + b];
      count += (uint32_t)(w >> kCountShift);
      less += w & kMask;
    }
    if (half == 1) {
      s.fine[b] = less;
      s.fine_counts[b] = count;
    }
    __syncthreads();
    if (half == 0) {
      less += s.fine[b];
      count += s.fine_counts[b];
    }
    const double base = 0x1p-40 * base_of(b);
    if (half == 0) s.base[b] = base;
    run_bins(s, base * ((double)count * 0x1p40 - (double)less), half == 0 ? count : 0u);
  }
  const int total = (int)s.counts[kSampleBins - 1];
  const double whole = s.sums[kSampleBins - 1];
  const Steps steps(top, temperature, s.table);
  Sampler<T> sampler{a, s, row, from, top, 11.541560327111707 / (double)temperature, steps};      // 8 / ln 2

  const int k = a.top_k == nullptr || a.top_k[row] <= 0 ? total : min(a.top_k[row], total);
  double p = a.top_p == nullptr ? 1.0 : (double)a.top_p[row], least = a.min_p == nullptr ? 0.0 : (double)a.min_p[row];
  if (!(least > 0.0)) least = 0.0;
  if (!(p < 1.0)) p = 1.0;
  const bool first_only = p <= 0.0 || least > 1.0;
  // Where the cut lies at most; where p is of the sum of the first k, all of those are wanted.  If a thread each is enough for the words up to there, they are sorted and the rest of the row is not looked at again.
  const int mine = min((int)threadIdx.x, kSampleBins - 1);
  const double my_sum = s.sums[mine];
  const uint32_t my_count = s.counts[mine];
  int bound = kSampleBins - 1;
  if (first_only || k < total) {
    find_bin(s, first_only ? 1u : (uint32_t)k, 0.0);
    bound = s.found;
    __syncthreads();
  }
  const bool all_of_k = k < total && p < 1.0;
  if (p < 1.0 && !first_only && !all_of_k) {
    find_bin(s, 0u, p * whole * (1.0 + 0x1p-30));
    bound = min(bound, s.found);
    __syncthreads();
  }
  if (least > 0.0 && !first_only && !all_of_k) bound = min(bound, max((int)(-log2f((float)least) * 8.f) + 1, 0));
  if (s.counts[bound] <= (uint32_t)kSampleThreads) {
    sampler.draw(bound, (int)s.counts[bound], first_only ? 1 : k, k < total ? -1.0 : whole, first_only ? 1.0 : p, first_only ? 0.0 : least);
    return;
  }

  if (threadIdx.x == 0) s.listed = 0;
  Cut cut{-INFINITY, 0x7fffffff};
  int last = kSampleBins - 1;      // the bin of the last word that stays, or a later one
  double part = whole;             // of the words in front of the first cut
  // first the cut behind so many words, then that behind so much of their sum.  (A bin's words share the space of the bins' running sums.)
#pragma unroll 1
  for (int stage = 0; stage < 2; ++stage) {
    const uint32_t count = stage > 0 ? 0u : first_only ? 1u : (uint32_t)k;
    if (stage == 0 ? !first_only && k >= total : first_only || p == 1.0) continue;
    __syncthreads();
    if (threadIdx.x < kSampleBins) {
      s.sums[threadIdx.x] = my_sum;
      s.counts[threadIdx.x] = my_count;
    }
    __syncthreads();
    find_bin(s, count, p * part);
    const int bin = s.found, before = s.before, words = (int)s.counts[bin] - before;
    const double front = s.sum_before;
    __syncthreads();
    const Cut next = sampler.cut_in(bin, words, count > 0 ? count - before : 0u, p * part - front);
    part = front + s.sum;
    if (next.at > cut.at || (next.at == cut.at && next.upto < cut.upto)) cut = next;      // the earlier of the two
    last = min(last, bin);
    __syncthreads();
  }
  // Bins in front of `near` stay as a whole and are known by chunks, those behind `far` go; the words between are looked at one by one, a chunk to a wavefront.
  int near = last, far = last;
  if (least > 0.0 && !first_only) {
    const int t = (int)fminf(-log2f((float)least) * 8.f, (float)kSampleBins);      // (or one beside it)
    near = max(min(near, t - 1), 0);
    far = min(far, t + 1);
  }
  const float low = fmaxf(sampler.lowest(far), cut.at), high = sampler.highest(near);
  // e of a word that stays, else 0
  auto e_if_kept = [&](float x, int i, int from) {
    const double y = steps.place(x);
    const int bin = steps.bin(y);
    if (bin < from || bin >= kSampleBins || !cut.has(x, i)) return 0.0;
    const double e = x == top ? 1.0 : sampler.e_at(y);
    return least == 0.0 || first_only || e >= least ? e : 0.0;
  };
  int kept = 0;
  // Words of the cut's step that LDS still has are added up from there, in 2^-51ths, so that their order does not matter.
  for (int c = threadIdx.x; c < a.chunks; c += kSampleThreads) s.chunks[c] = 0;
  __syncthreads();
  const bool held = s.listed > 0 && s.listed_bin == last && near == last && far == last;
  if (held)
    for (int j = threadIdx.x; j < s.listed; j += kSampleThreads) {
      const int i = (int)(uint32_t)s.list[j];
      const double e = e_if_kept(sampler.listed_logit(j), i, near);
      if (e > 0.0) atomicAdd(&s.chunks[(i + Chunk<T>::lead(from)) / Chunk<T>::kElements], (unsigned long long)__builtin_rint(e * 0x1p51));
      kept += e > 0.0;
    }
  __syncthreads();
  for (int c = wave; c < a.chunks; c += kSampleWaves) {
    double sum = lane == 0 ? (double)s.chunks[c] * 0x1p-51 : 0.0;
    bool any = false;
    unsigned long long w[kSampleBins / 64];
#pragma unroll
    for (int j = 0; j < kSampleBins / 64; ++j) w[j] = bins[(int64_t)c * kSampleBins + 64 * j + lane];
#pragma unroll
    for (int j = 0; j < kSampleBins / 64; ++j) {
      any = any || (64 * j + lane >= near && 64 * j + lane <= far && w[j] != 0);
      if (64 * j + lane >= near) continue;
      kept += (int)(w[j] >> kCountShift);
      sum += s.base[64 * j + lane] * ((double)(w[j] >> kCountShift) * 0x1p40 - (double)(w[j] & kMask));
    }
    if (!held && __any(any))
      each_piece<T>(from, a.vocabulary, c * Chunk<T>::kElements - Chunk<T>::lead(from), Chunk<T>::kElements / Chunk<T>::E, lane, 64, [&](const typename Piece<T>::type& v, int i) {
        each_between<T>(v, i, low, high, [&](float x, int at) {
          const double e = e_if_kept(x, at, near);
          sum += e;
          kept += e > 0.0;
        });
      });
    sum = wave_sum(sum);
    if (lane == 0) s.chunks[c] = __builtin_bit_cast(unsigned long long, sum);
  }
  __syncthreads();
  if (threadIdx.x == 0) s.before = 0;
  __syncthreads();
  kept = (int)wave_sum((double)kept);
  if (lane == 0) atomicAdd(&s.before, kept);
  // the chunk of the word: two chunks to a thread
  double pair[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) pair[j] = 2 * (int)threadIdx.x + j < a.chunks ? __builtin_bit_cast(double, (uint64_t)s.chunks[2 * threadIdx.x + j]) : 0.0;
  double upto = group_scan(s, pair[0] + pair[1]);
  const double all = of_waves(s, kSampleWaves), want = (double)a.uniforms[row] * all;
  if (threadIdx.x == 0) {
    s.found = 0x7fffffff;
    s.length = -1;      // the last chunk with a word
  }
  __syncthreads();
#pragma unroll
  for (int j = 1; j >= 0; --j) {
    if (pair[j] > 0.0) {
      atomicMax(&s.length, 2 * (int)threadIdx.x + j);
      if ((j == 0 ? upto - pair[1] : upto) > want) atomicMin(&s.found, 2 * (int)threadIdx.x + j);
    }
  }
  __syncthreads();
  const int chunk = min(s.found, s.length);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 2; ++j)
    if (2 * (int)threadIdx.x + j == chunk) s.sum_before = upto - pair[1] - (j == 0 ? pair[0] : 0.0);
  if (threadIdx.x == 0) {
    s.found = 0x7fffffff;
    s.length = -1;      // the last thread with one
  }
  __syncthreads();
  constexpr int EACH = Chunk<T>::kElements / kSampleThreads;
  const int first = chunk * Chunk<T>::kElements + EACH * (int)threadIdx.x - Chunk<T>::lead(from);
  static_assert(EACH == Chunk<T>::E, "a piece to a thread");
  const typename Piece<T>::type x = piece_at<T>(from, a.vocabulary, first);
  double e[EACH], sum = 0.0;
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    e[j] = e_if_kept((float)x[j], first + j, 0);
    sum += e[j];
  }
  upto = s.sum_before + group_scan(s, sum);
  if (sum > 0.0) {
    atomicMax(&s.length, (int)threadIdx.x);
    if (upto > want) atomicMin(&s.found, (int)threadIdx.x);
  }
  __syncthreads();
  if ((int)threadIdx.x != min(s.found, s.length)) return;      // (rounding may leave the sum short of its whole: then it is the last that stays)
  double run = upto - sum;
  int word = -1;
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    if (e[j] > 0.0 && !(word >= 0 && run > want)) word = first + j;
    run += e[j];
  }
  a.words[row] = word;
  if (a.kept != nullptr) a.kept[row] = s.before;
}

}  // namespace dpllm
