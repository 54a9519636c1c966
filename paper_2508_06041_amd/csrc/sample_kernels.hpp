// A word for every row of logits.  e = exp((x - top) / temperature); the words in the order of their logits (equal ones by number) are cut off behind the first top_k, where less than
// top_p of the sum of those lies in front, and at e = min_p: all three leave the first so many of one order.  So nothing is sorted: a histogram of the row over
// eighths of a power of two of e says in which step of it a cut lies, and only the words of that step are looked at one by one.
//
// Answers are whole numbers, so sums are kept in 64 bits and in whole numbers where workgroups' order could show: a word of step b counts 1 and the
// 2^-40ths by which e 2^((b + 1) / 8) exceeds 1, both in one 64-bit addition in LDS.  Rounding that to 2^-41 moves a sum by less than 1e-12 of itself.
#pragma once
#include "verify_kernels.hpp"

namespace dpllm {

constexpr int kSampleBins = 512;            // e down to 2^-64
constexpr int kSampleThreads = 1024;        // of the workgroup that chooses
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kSampleList = 2048;           // words that are sorted at once
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

// Where a word lies: eighths of a power of two below the top, by = 8 / (temperature ln 2).  false: it is left out (as are NaN and minus infinity).
__device__ __forceinline__ bool step_of(float x, float top, double by, int* bin, double* part) {
  const double t = x == top ? 0.0 : ((double)top - (double)x) * by;
  if (!(t <= (double)kSampleBins)) return false;
  *bin = min((int)t, kSampleBins - 1);
  *part = t - (double)*bin;
  return true;
}
// 2^((1 - part) / 8) - 1 in 2^-40ths: the series to its eighth power, below 1e-15.
__device__ __forceinline__ unsigned long long excess(double part) {
  const double y = (1.0 - part) * 0.086643397569993164;      // ln 2 / 8
  double s = 1.0 / 40320.0;
  s = __builtin_fma(s, y, 1.0 / 5040.0);
  s = __builtin_fma(s, y, 1.0 / 720.0);
  s = __builtin_fma(s, y, 1.0 / 120.0);
  s = __builtin_fma(s, y, 1.0 / 24.0);
  s = __builtin_fma(s, y, 1.0 / 6.0);
  s = __builtin_fma(s, y, 0.5);
  s = __builtin_fma(s, y, 1.0);
  return (unsigned long long)__builtin_rint(s * y * 0x1p40);
}
__device__ __forceinline__ double steps_by(float temperature) { return 11.541560327111707 / (double)temperature; }      // 8 / ln 2
__device__ __forceinline__ double base_of(int bin) { return exp_of(-0.086643397569993164 * (bin + 1)); }
__device__ __forceinline__ float larger(float x, float y) { return fmaxf(x, y); }
__device__ __forceinline__ int smaller(int x, int y) { return min(x, y); }

// The largest logit of a chunk.
template <typename T>
__global__ void __launch_bounds__(kVerThreads) sample_tops_kernel(const SampleArgs a, const Divide by_chunks) {
  __shared__ float tops[kVerThreads / 64];
  __shared__ int places[kVerThreads / 64];
  const int row = by_chunks.of(blockIdx.x), chunk = blockIdx.x - row * a.chunks;
  const char* from = a.logits + row * a.stride * (int64_t)sizeof(T);
  Chunk<T> c;
  c.load(from, chunk, a.vocabulary);
  float top = -INFINITY;
#pragma unroll
  for (int p = 0; p < kVerPieces; ++p)
#pragma unroll
    for (int e = 0; e < Chunk<T>::E; ++e) top = fmaxf(top, c.x[p][e]);
  top = wave_all(top, larger);
  int at = 0x7fffffff;
#pragma unroll
  for (int p = 0; p < kVerPieces; ++p)
#pragma unroll
    for (int e = 0; e < Chunk<T>::E; ++e)
      if (c.x[p][e] == top && top != -INFINITY) at = min(at, Chunk<T>::index(from, chunk, p, e));
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
__global__ void __launch_bounds__(kVerThreads) sample_bins_kernel(const SampleArgs a, const Divide by_chunks) {
  __shared__ unsigned long long bins[kSampleBins];
  const int row = by_chunks.of(blockIdx.x), chunk = blockIdx.x - row * a.chunks;
  const float temperature = a.temperature[row];
  if (greedy(temperature)) return;
  const char* from = a.logits + row * a.stride * (int64_t)sizeof(T);
  Chunk<T> c;
  c.load(from, chunk, a.vocabulary);
  for (int i = threadIdx.x; i < kSampleBins; i += kVerThreads) bins[i] = 0;
  float top = -INFINITY;
  for (int i = threadIdx.x & 63; i < a.chunks; i += 64) top = fmaxf(top, a.tops[(int64_t)row * a.chunks + i].top);
  top = wave_all(top, larger);
  __syncthreads();
  if (top == -INFINITY) return;
  const double by = steps_by(temperature);
#pragma unroll
  for (int p = 0; p < kVerPieces; ++p)
#pragma unroll
    for (int e = 0; e < Chunk<T>::E; ++e) {
      int bin;
      double part;
      // (what lies outside of the row is minus infinity)
      if (step_of(c.x[p][e], top, by, &bin, &part)) atomicAdd(&bins[bin], (1ull << kCountShift) + excess(part));
    }
  __syncthreads();
  for (int i = threadIdx.x; i < kSampleBins; i += kVerThreads) a.bins[((int64_t)row * a.chunks + chunk) * kSampleBins + i] = bins[i];
}

// Words in front of a cut: those above its logit, and of those at it the ones up to a number.
struct Cut {
  float at;
  int upto;
  __device__ __forceinline__ bool has(float x, int i) const { return x > at || (x == at && i <= upto); }
};

// Floats as whole numbers in the same order (-0 and 0 are one).
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t w = __float_as_uint(x + 0.f);
  return w >> 31 ? ~w : w | 0x80000000u;
}
__device__ __forceinline__ float from_key(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

struct SampleSpace {
  unsigned long long list[kSampleList];
  double sums[kSampleBins];                 // running, over bins
  uint32_t counts[kSampleBins];
  unsigned long long fine[kSampleBins];     // of a step that is looked at more closely
  uint32_t fine_counts[kSampleBins];
  double wave_sums[kSampleWaves];
  uint32_t wave_counts[kSampleWaves];
  double sum, sum_before;
  int found, before, length;
  uint32_t low, high;
};

// The running sums of kSampleBins values and counts, one of each to a thread of the first eight wavefronts, into s.sums and s.counts.
__device__ __forceinline__ void run_bins(SampleSpace& s, double sum, uint32_t count) {
  const int wave = threadIdx.x >> 6;
  const double upto = wave_scan(sum), number = wave_scan((double)count);      // (whole numbers)
  __syncthreads();
  if ((threadIdx.x & 63) == 63 && threadIdx.x < kSampleBins) {
    s.wave_sums[wave] = upto;
    s.wave_counts[wave] = (uint32_t)number;
  }
  __syncthreads();
  if (threadIdx.x < kSampleBins) {
    double plus = 0.0;
    uint32_t more = 0;
    for (int w = 0; w < wave; ++w) {
      plus += s.wave_sums[w];
      more += s.wave_counts[w];
    }
    s.sums[threadIdx.x] = upto + plus;
    s.counts[threadIdx.x] = (uint32_t)number + more;
  }
  __syncthreads();
}

// The first bin up to which there are `count` words, or (count 0) a sum of `sum`; the last one with a word if there is none.  s.found, s.before and s.sum_before: what lies in front.
__device__ __forceinline__ void find_bin(SampleSpace& s, uint32_t count, double sum) {
  const int b = threadIdx.x;
  if (b < kSampleBins) {
    const uint32_t upto = s.counts[b], front = b == 0 ? 0u : s.counts[b - 1], all = s.counts[kSampleBins - 1];
    const double s_upto = s.sums[b], s_front = b == 0 ? 0.0 : s.sums[b - 1];
    const bool here = count > 0 ? upto >= count : s_upto >= sum, there = b > 0 && (count > 0 ? front >= count : s_front >= sum);
    const bool last = upto == all && front < all;      // (rounding may leave a sum short of its whole)
    const bool none = count > 0 ? all < count : s.sums[kSampleBins - 1] < sum;
    if (none ? last : here && !there) {
      s.found = b;
      s.before = (int)front;
      s.sum_before = s_front;
    }
  }
  __syncthreads();
}

// f(x, i) for those of a piece of a row that are within [low, high].  They are few, or dear: so f's code is there once, and they are read again.
template <typename T, typename F>
__device__ __forceinline__ void each_between(const typename Piece<T>::type& v, const char* row, int first, float low, float high, F f) {
  uint32_t in = 0;
#pragma unroll
  for (int e = 0; e < Piece<T>::E; ++e) in |= (float)v[e] >= low && (float)v[e] <= high ? 1u << e : 0u;
#pragma unroll 1
  while (in != 0) {
    const int i = first + __builtin_ctz(in);
    f(logit<T>(row, i), i);
    in &= in - 1;
  }
}

// f(x, i) for all words of a row whose logits are within [low, high], in no order.
template <typename T, typename F>
__device__ __forceinline__ void words_between(const char* row, int n, float low, float high, F f) {
  constexpr int E = Piece<T>::E;
  typedef typename Piece<T>::type piece;
  const int lead = Chunk<T>::lead(row), pieces = (n + lead + E - 1) / E;
  const T* base = reinterpret_cast<const T*>(row);
  for (int p0 = threadIdx.x; p0 < pieces; p0 += 4 * kSampleThreads) {
    piece v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = (p0 + j * kSampleThreads) * E - lead;
      if (i >= 0 && i + E <= n) {
        v[j] = *reinterpret_cast<const piece*>(base + i);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[j][e] = i + e >= 0 && i + e < n ? base[i + e] : (T)__builtin_nanf("");
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) each_between<T>(v[j], row, (p0 + j * kSampleThreads) * E - lead, low, high, f);
  }
}

// Sorts n (a power of two) numbers, the smallest first.
__device__ __forceinline__ void sort(unsigned long long* list, int n) {
  for (int size = 2; size <= n; size *= 2)
    for (int gap = size / 2; gap > 0; gap /= 2) {
      for (int i = threadIdx.x; i < n / 2; i += kSampleThreads) {
        const int p = 2 * i - (i & (gap - 1)), q = p + gap;
        const unsigned long long x = list[p], y = list[q];
        if ((x > y) == ((p & size) == 0)) {
          list[p] = y;
          list[q] = x;
        }
      }
      __syncthreads();
    }
}

// The running sum over the workgroup of a value of each thread.
__device__ __forceinline__ double group_scan(SampleSpace& s, double v) {
  const int wave = threadIdx.x >> 6;
  double upto = wave_scan(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) s.wave_sums[wave] = upto;
  __syncthreads();
  double plus = 0.0;
  for (int w = 0; w < wave; ++w) plus += s.wave_sums[w];
  return upto + plus;
}

// The order of the row as its histogram's bins are; all threads take part in each of these.
template <typename T>
struct Sampler {
  const SampleArgs& a;
  SampleSpace& s;
  const char* row;
  float top;
  double by, inverse;      // steps and 1 / temperature

  __device__ __forceinline__ double e_of(float x) const { return weight(x, top, inverse); }
  // Bounds of the logits of bins first ... last, a little wide.
  __device__ __forceinline__ float lowest(int last) const {
    const float x = (float)((double)top - (last + 1) / by);
    if (top == INFINITY) return top;
    return x != x || last >= kSampleBins - 1 ? -INFINITY : x - __builtin_fabsf(x) * 0x1p-20f - 0x1p-120f;
  }
  __device__ __forceinline__ float highest(int first) const {
    const float x = (float)((double)top - first / by);
    return first == 0 || x != x ? INFINITY : x + __builtin_fabsf(x) * 0x1p-20f + 0x1p-120f;
  }

  // The words of bin `bin` in front of a cut: `count` of them, or (count 0) those in front of which less than `sum` of them lies, at least one.  s.length and s.sum: how many, and their sum.
  __device__ Cut cut_in(int bin, int words, uint32_t count, double sum) {
    uint32_t low = 0, high = ~0u;      // keys
    const double base = base_of(bin);
    int taken = 0;
    double taken_sum = 0.0;
    const auto inside = [&](float x, double* part) {
      int b;
      const uint32_t k = key_of(x);
      return k >= low && k <= high && step_of(x, top, by, &b, part) && b == bin;
    };
    // narrower, until the words can be sorted or are all the same: nine of the key's 32 bits at a time
    for (int round = 0; round < 4 && words > kSampleList && low != high; ++round) {
      if (threadIdx.x == 0) {
        s.low = ~0u;
        s.high = 0u;
      }
      if (threadIdx.x < kSampleBins) {
        s.fine[threadIdx.x] = 0;
        s.fine_counts[threadIdx.x] = 0;
      }
      __syncthreads();
      uint32_t least = ~0u, most = 0u;
      words_between<T>(row, a.vocabulary, lowest(bin), highest(bin), [&](float x, int) {
        double part;
        if (inside(x, &part)) {
          least = min(least, key_of(x));
          most = max(most, key_of(x));
        }
      });
      least = wave_all(least, [](uint32_t x, uint32_t y) { return min(x, y); });
      most = wave_all(most, [](uint32_t x, uint32_t y) { return max(x, y); });
      if ((threadIdx.x & 63) == 0) {
        atomicMin(&s.low, least);
        atomicMax(&s.high, most);
      }
      __syncthreads();
      low = s.low;
      high = s.high;
      if (low == high) break;
      const int shift = max(0, 23 - __builtin_clz(high - low));      // (high - low) >> shift is below 512
      words_between<T>(row, a.vocabulary, lowest(bin), highest(bin), [&](float x, int) {
        double part;
        if (inside(x, &part)) {
          atomicAdd(&s.fine_counts[(high - key_of(x)) >> shift], 1u);
          atomicAdd(&s.fine[(high - key_of(x)) >> shift], excess(part));
        }
      });
      __syncthreads();
      const int i = min((int)threadIdx.x, kSampleBins - 1);
      run_bins(s, base * ((double)s.fine_counts[i] + (double)s.fine[i] * 0x1p-40), s.fine_counts[i]);
      find_bin(s, count > 0 ? count - taken : 0u, sum - taken_sum);
      taken += s.before;
      taken_sum += s.sum_before;
      words = (int)(s.counts[s.found] - s.before);
      const uint32_t upper = high - ((uint32_t)s.found << shift), width = (1u << shift) - 1u;
      low = max(low, upper - min(upper, width));
      high = upper;
      __syncthreads();
    }
    if (words <= kSampleList) {
      if (threadIdx.x == 0) s.length = 0;
      int size = 2;
      while (size < words) size *= 2;
      for (int i = threadIdx.x; i < size; i += kSampleThreads) s.list[i] = ~0ull;
      __syncthreads();
      words_between<T>(row, a.vocabulary, lowest(bin), highest(bin), [&](float x, int i) {
        double part;
        if (inside(x, &part)) {
          const int at = atomicAdd(&s.length, 1);
          if (at < kSampleList) s.list[at] = (unsigned long long)~key_of(x) << 32 | (uint32_t)i;
        }
      });
      __syncthreads();
      sort(s.list, size);
      // two words to a thread
      const int i = 2 * threadIdx.x;
      double e[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) e[j] = i + j < words ? e_of(from_key(~(uint32_t)(s.list[i + j] >> 32))) : 0.0;
      const double upto = group_scan(s, e[0] + e[1]);
      if (threadIdx.x == 0) s.found = -1;
      __syncthreads();
      int last = -1;      // the last of this thread's that stays
      double last_sum = 0.0;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const double front = upto - (j == 0 ? e[0] + e[1] : e[1]);
        if (i + j < words && (count > 0 ? (uint32_t)(taken + i + j) < count : i + j + taken == 0 || taken_sum + front < sum)) {
          last = i + j;
          last_sum = front + e[j];
        }
      }
      atomicMax(&s.found, last);
      __syncthreads();
      if (last >= 0 && last == s.found) s.sum = taken_sum + last_sum;
      const int found = max(s.found, 0);
      if (threadIdx.x == 0) {
        s.length = taken + s.found + 1;
        if (s.found < 0) s.sum = taken_sum;
      }
      const unsigned long long w = s.list[found];
      __syncthreads();
      // (rounding between two ways to the same sum may leave none of these: then the cut is in front of the first)
      if (s.length == taken) return {from_key(~(uint32_t)(w >> 32)), -1};
      return {from_key(~(uint32_t)(w >> 32)), (int)(uint32_t)w};
    }
    // all the same: so many of them by their numbers
    const float x = from_key(high);
    const double e = e_of(x);
    int n = count > 0 ? (int)count - taken : (int)fmin((sum - taken_sum) / e, (double)words);
    if (count == 0) {
      while (n > 0 && (n - 1) * e >= sum - taken_sum) --n;
      while (n < words && n * e < sum - taken_sum) ++n;
    }
    n = min(max(n, 1), words);
    int upto = 0x7fffffff;
    if (n < words) {
      // the n-th by number: a stretch of the row at a time
      int seen = 0;
      for (int first = 0; first < a.vocabulary; first += 8 * kSampleThreads) {
        int mine = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = first + 8 * threadIdx.x + j;
          mine += i < a.vocabulary && logit<T>(row, i) == x;
        }
        const int before = (int)group_scan(s, (double)mine) - mine;
        if (seen + before < n && n <= seen + before + mine) {
          int k = seen + before;
#pragma unroll 1
          for (int j = 0; j < 8; ++j) {
            const int i = first + 8 * threadIdx.x + j;
            if (i < a.vocabulary && logit<T>(row, i) == x && ++k == n) s.found = i;
          }
        }
        int all = 0;
        for (int w = 0; w < kSampleWaves; ++w) all += (int)s.wave_sums[w];
        seen += all;
        __syncthreads();
        if (seen >= n) {
          upto = s.found;
          break;
        }
      }
    }
    if (threadIdx.x == 0) {
      s.length = taken + n;
      s.sum = taken_sum + n * e;
    }
    __syncthreads();
    return {x, upto};
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
    const int b = threadIdx.x & (kSampleBins - 1), half = threadIdx.x / kSampleBins;
    uint32_t count = 0;
    unsigned long long more = 0;
    for (int c = half; c < a.chunks; c += 2) {
      const unsigned long long w = bins[(int64_t)c * kSampleBins + b];
      count += (uint32_t)(w >> kCountShift);
      more += w & kMask;
    }
    if (half == 1) {
      s.fine[b] = more;
      s.fine_counts[b] = count;
    }
    __syncthreads();
    if (half == 0) {
      more += s.fine[b];
      count += s.fine_counts[b];
    }
    run_bins(s, base_of(b) * ((double)count + (double)more * 0x1p-40), half == 0 ? count : 0u);
  }
  const int total = (int)s.counts[kSampleBins - 1];
  const double whole = s.sums[kSampleBins - 1];
  Sampler<T> sampler{a, s, from, top, steps_by(temperature), 1.0 / (double)temperature};

  const int k = a.top_k == nullptr || a.top_k[row] <= 0 ? total : min(a.top_k[row], total);
  double p = a.top_p == nullptr ? 1.0 : (double)a.top_p[row], least = a.min_p == nullptr ? 0.0 : (double)a.min_p[row];
  if (!(least > 0.0)) least = 0.0;
  const bool first_only = p <= 0.0 || least > 1.0;
  Cut cut{-INFINITY, 0x7fffffff};
  int last = kSampleBins - 1;      // the bin of the last word that stays, or a later one
  double part = whole;             // of the words in front of the first cut
  // first the cut behind so many words, then that behind so much of their sum.  (A bin's words share the space of the bins' running sums.)
  const int mine = min((int)threadIdx.x, kSampleBins - 1);
  const double my_sum = s.sums[mine];
  const uint32_t my_count = s.counts[mine];
#pragma unroll 1
  for (int stage = 0; stage < 2; ++stage) {
    const uint32_t count = stage > 0 ? 0u : first_only ? 1u : (uint32_t)k;
    if (stage == 0 ? !first_only && k >= total : first_only || !(p < 1.0)) continue;
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
  if (least > 0.0) {
    const float t = -log2f((float)least) * 8.f;
    if (t < (float)last) last = max((int)t, 0);
  }

  // Bins that stay as a whole are known by chunks; those around the cut are looked at word by word, a chunk to a wavefront.
  const int near = max(last - 1, 0), far = min(last + 1, kSampleBins - 1);
  const float low = sampler.lowest(far), high = sampler.highest(near);
  auto stays = [&](float x, int i, int* bin) {
    double rest;
    return step_of(x, top, sampler.by, bin, &rest) && cut.has(x, i) && (least == 0.0 || first_only || sampler.e_of(x) >= least);
  };
  double* chunk_sums = reinterpret_cast<double*>(s.list);      // [up to kSampleList chunks]
  int kept = 0;
  __syncthreads();
  for (int c = wave; c < a.chunks; c += kSampleWaves) {
    double sum = 0.0;
    for (int b = lane; b < near; b += 64) {
      const unsigned long long w = bins[(int64_t)c * kSampleBins + b];
      kept += (int)(w >> kCountShift);
      sum += base_of(b) * ((double)(w >> kCountShift) + (double)(w & kMask) * 0x1p-40);
    }
    constexpr int E = Piece<T>::E;
    typedef typename Piece<T>::type piece;
    const T* words = reinterpret_cast<const T*>(from);
    for (int q = lane; q < Chunk<T>::kElements / E; q += 64) {
      const int i = c * Chunk<T>::kElements + q * E - Chunk<T>::lead(from);
      piece v;
      if (i >= 0 && i + E <= a.vocabulary) {
        v = *reinterpret_cast<const piece*>(words + i);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = i + e >= 0 && i + e < a.vocabulary ? words[i + e] : (T)__builtin_nanf("");
      }
      each_between<T>(v, from, i, low, high, [&](float x, int at) {
        int bin;
        if (stays(x, at, &bin) && bin >= near) {
          sum += sampler.e_of(x);
          ++kept;
        }
      });
    }
    sum = wave_sum(sum);
    if (lane == 0) chunk_sums[c] = sum;
  }
  __syncthreads();
  kept = (int)wave_sum((double)kept);
  if (lane == 0) s.wave_counts[wave] = (uint32_t)kept;
  // the chunk of the word: two chunks to a thread
  double pair[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) pair[j] = 2 * (int)threadIdx.x + j < a.chunks ? chunk_sums[2 * threadIdx.x + j] : 0.0;
  double upto = group_scan(s, pair[0] + pair[1]);
  double all = 0.0;
  for (int w = 0; w < kSampleWaves; ++w) all += s.wave_sums[w];
  const double want = (double)a.uniforms[row] * all;
  if (threadIdx.x == 0) {
    s.found = 0x7fffffff;
    s.length = -1;      // the last chunk with a word
    uint32_t n = 0;
    for (int w = 0; w < kSampleWaves; ++w) n += s.wave_counts[w];
    if (a.kept != nullptr) a.kept[row] = (int)n;
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
  auto e_at = [&](int i) {
    if (i < 0 || i >= a.vocabulary) return 0.0;
    const float x = logit<T>(from, i);
    int bin;
    return stays(x, i, &bin) ? sampler.e_of(x) : 0.0;
  };
  double sum = 0.0;
#pragma unroll 1
  for (int j = 0; j < EACH; ++j) sum += e_at(first + j);
  upto = s.sum_before + group_scan(s, sum);
  if (sum > 0.0) {
    atomicMax(&s.length, (int)threadIdx.x);
    if (upto > want) atomicMin(&s.found, (int)threadIdx.x);
  }
  __syncthreads();
  if ((int)threadIdx.x != min(s.found, s.length)) return;      // (rounding may leave the sum short of its whole: then it is the last that stays)
  double run = upto - sum;
  int word = -1;
#pragma unroll 1
  for (int j = 0; j < EACH; ++j) {
    const double e = e_at(first + j);
    run += e;
    if (e > 0.0) word = first + j;
    if (e > 0.0 && run > want) break;
  }
  a.words[row] = word;
}

}  // namespace dpllm
