// Verification of drafted tokens.  p_i = softmax(logits_i / temperature) and q_i = softmax(draft_i / temperature) of node i.  The children c of a node, in the
// order of their numbers, are taken with probability min(1, r(c) / q(c)), r = p at first, and r <- max(r - q, 0) / (its sum) behind a child that was
// not.  All those r have one form: r_j = max(p - a_j q, 0) / S_j, a_0 = 0, S_0 = 1, a_(j+1) = a_j + S_j, S_j = sum of max(p - a_j q, 0) (with
// r_j = max(p - a_j q, 0) / S_j, r_j - q is (p - a_j q - S_j q) / S_j where that is positive), so a row's state is two numbers and one more
// sum over the row moves it on.  Without draft rows a child was named, not drawn, and leaves the distribution when it is not taken.
//
// Answers are whole numbers, so nothing may hang on the order of additions: logits are widened, and differences, exponentials and sums are kept, in
// 64 bits; two orders of a sum of 10^5 terms differ by about 1e-14, and so do the numbers that a probability of 2^-24 steps is compared with.
#pragma once
#include "lanes.hpp"
#include "token_common.hpp"

namespace dpllm {

constexpr int kVerThreads = 256;
constexpr int kVerPieces = 4;                                 // 16-byte pieces of a row to a thread
constexpr int kVerMaxNodes = DPLLM_MAX_NODES;

struct VerifyPart {      // of a chunk of a row: its largest logit, where that is first, the sum of exp((x - top) / temperature)
  double sum;
  float top;
  int at;
};

struct RowInfo;
struct VerifyArgs {
  const char *logits, *draft;
  int64_t logits_batch, logits_node, draft_batch, draft_node;      // elements
  const int32_t *tokens, *parents;
  const float *uniforms, *temperature;
  int32_t *count, *path, *words;
  VerifyPart* parts;       // [2 with draft rows][batch * nodes][chunks]
  double* rest;            // [siblings][batch * nodes][chunks]: sums of max(p - a q, 0)
  RowInfo* infos;   // [batch * nodes] with draft rows
  int batch, nodes, vocabulary, chunks, siblings;
};

// 2^(t - rint(t)) by the series of exp to its eleventh power (below 1e-14 for arguments up to ln 2 / 2), times 2^rint(t).  y = 0 gives exactly 1;
// -infinity and NaN give 0.
__device__ __forceinline__ double exp_of(double y) {
  const double t = __builtin_fmax(y * 1.4426950408889634074, -1100.0);
  const double n = __builtin_rint(t), x = (t - n) * 0.69314718055994530942;
  double s = 1.0 / 39916800.0;
  s = __builtin_fma(s, x, 1.0 / 3628800.0);
  s = __builtin_fma(s, x, 1.0 / 362880.0);
  s = __builtin_fma(s, x, 1.0 / 40320.0);
  s = __builtin_fma(s, x, 1.0 / 5040.0);
  s = __builtin_fma(s, x, 1.0 / 720.0);
  s = __builtin_fma(s, x, 1.0 / 120.0);
  s = __builtin_fma(s, x, 1.0 / 24.0);
  s = __builtin_fma(s, x, 1.0 / 6.0);
  s = __builtin_fma(s, x, 0.5);
  s = __builtin_fma(s, x, 1.0);
  s = __builtin_fma(s, x, 1.0);
  return __builtin_ldexp(s, (int)n);
}

// exp((x - top) / temperature); the largest counts 1 also where it is infinite, and a row without a number (top is -infinity) has no weight
__device__ __forceinline__ double weight(float x, float top, double by) {
  if (top == -INFINITY) return 0.0;
  return x == top ? 1.0 : exp_of(((double)x - (double)top) * by);
}

// The same for the sums over many logits of one row, without a branch, in few instructions, as these are what the sums are bound by.  (x - top) / temperature is
// counted in 256ths of a power of two from 2^19 - 256, so that all that come up lie between 2^18 and 2^19: the last two bits of the upper word and the
// lower word are the fraction r, the eight before them the place in a table of 2^(j / 256) in LDS, and those before the power of two.  1 + c1 r + c2 r^2 + c3 r^3 is
// 2^(r / 256) to 2e-14, with the largest such error made least and none at 0, so that the largest logit counts exactly 1; the count is rounded to 2^-34, which is
// 8e-14 of a weight at most.  With a count that is rounded to the nearest whole and the series to the fourth power (1e-15; three instructions in
// twenty more) verify_parts took 69 us for 48 sequences of 8 nodes with draft rows of 128256 words in bf16 (16 of the sequences take the best token: 66 million
// weights), with this 60, and 54 since a workgroup takes several chunks of a row.
// Logits more than 690 temperatures below the largest, minus infinities and NaN among them, count as the one that is, whose weight of
// 1e-300 is nothing to a sum.  A row whose largest logit is no finite number, or beside which 695 temperatures are
// past the floats or lost in their rounding, goes the way above.
constexpr int kVerTable = 256;      // entries: their lower words, then their upper ones, so that both are one read
struct Weigher {
  const uint32_t* table;
  double top, steps;
  float least;
  bool plain;
  __device__ __forceinline__ Weigher(const uint32_t* table, float top, double by)
      : table(table), top((double)top), steps(by * 369.32993046757462), least((float)((double)top - 695.0 / by)) {      // 256 / ln 2
    const double below = ((double)top - (double)least) * by;      // 695, but for the rounding of a float
    plain = __builtin_isfinite(top) && below > 690.0 && below < 700.0;
  }
  // The weight is g * f.  The logit is no signaling NaN (a Chunk's never are), so that one instruction takes the larger.
  __device__ __forceinline__ void parts(float x, double& g, double& f) const {
    float z;
    asm("v_max_f32 %0, %1, %2" : "=v"(z) : "v"(x), "v"(least));
    const double y = __builtin_fma((double)z - top, steps, 524032.0), r = __builtin_amdgcn_fract(y);      // 2^19 - 256
    const uint32_t i = (uint32_t)(__builtin_bit_cast(uint64_t, y) >> 32);
    const uint32_t* at = reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(table) + (i & (4 * kVerTable - 4)));
    uint32_t high;
    asm("v_lshl_add_u32 %0, %1, 10, %2" : "=v"(high) : "v"(i & ~(4 * kVerTable - 1u)), "v"(at[kVerTable]));
    g = __builtin_bit_cast(double, (uint64_t)high << 32 | at[0]);
    f = __builtin_fma(r, 3.312607527945956e-09, 3.6655631008313955e-06);
    f = __builtin_fma(f, r, 0.0027076061744736664);
    f = __builtin_fma(f, r, 1.0);
  }
  __device__ __forceinline__ double of(float x) const {
    double g, f;
    parts(x, g, f);
    return g * f;
  }
  __device__ __forceinline__ double plus(float x, double sum) const {
    double g, f;
    parts(x, g, f);
    return __builtin_fma(g, f, sum);
  }
};
// Fills the table; a barrier has to follow.  The largest logit's count leaves 0x7ff00000 of the power of two's place, which is taken off here.
__device__ __forceinline__ void fill_table(uint32_t* table) {
  for (int i = threadIdx.x; i < kVerTable; i += blockDim.x) {
    const uint64_t w = __builtin_bit_cast(uint64_t, exp_of(i * 0.0027076061740622863));      // ln 2 / 256
    table[i] = (uint32_t)w;
    table[kVerTable + i] = (uint32_t)(w >> 32) - 0x7ff00000u;
  }
}

// The temperature of a sequence: 0 (or less, or NaN) takes the best token.
__device__ __forceinline__ bool greedy(float temperature) { return !(temperature > 0.f); }

// NaN counts as minus infinity.
__device__ __forceinline__ float number(float x) { return x == x ? x : -INFINITY; }

template <typename T>
__device__ __forceinline__ float logit(const char* row, int i) { return (float)reinterpret_cast<const T*>(row)[i]; }

// A chunk of a row in registers: piece p of a thread is the 16 bytes (p * threads + thread) of the chunk, counted from the last 16-byte boundary in front
// of the row.  Pieces that the row covers in part are read element by element; what lies outside is -infinity.  NaN are quiet.
template <typename T>
struct Chunk {
  static constexpr int E = Piece<T>::E;
  static constexpr int kElements = kVerThreads * kVerPieces * E;
  float x[kVerPieces][E];
  __device__ __forceinline__ static int lead(const char* row) { return (int)((uintptr_t)row % 16 / sizeof(T)); }
  // the number in the row of element e of piece p
  __device__ __forceinline__ static int index(const char* row, int chunk, int p, int e) {
    return chunk * kElements + (p * kVerThreads + (int)threadIdx.x) * E + e - lead(row);
  }
  // on its way from memory
  struct Raw {
    typename Piece<T>::type v[kVerPieces];
    __device__ __forceinline__ void load(const char* row, int chunk, int n) {
      const T* base = reinterpret_cast<const T*>(row);
#pragma unroll
      for (int p = 0; p < kVerPieces; ++p) {
        const int i = index(row, chunk, p, 0);
        if (i >= 0 && i + E <= n) {
          v[p] = *reinterpret_cast<const typename Piece<T>::type*>(base + i);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) v[p][e] = i + e >= 0 && i + e < n ? base[i + e] : (T)-INFINITY;
        }
      }
    }
  };
  __device__ __forceinline__ void take(const Raw& raw) {
#pragma unroll
    for (int p = 0; p < kVerPieces; ++p)
#pragma unroll
      for (int e = 0; e < E; ++e) x[p][e] = __builtin_canonicalizef((float)raw.v[p][e]);
  }
  __device__ __forceinline__ void load(const char* row, int chunk, int n) {
    Raw raw;
    raw.load(row, chunk, n);
    take(raw);
  }
};

// The value of one lane, which is the same for all.
__device__ __forceinline__ double of_lane(double v, int lane) {
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  const uint32_t low = __builtin_amdgcn_readlane((int)(uint32_t)w, lane), high = __builtin_amdgcn_readlane((int)(uint32_t)(w >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}

// The sum over this lane and those before it: inside sixteen lanes by shifts, then the last of a sixteen is added to the next sixteen and the last of the
// first half to the second.  A lane that has no source adds 0.
template <int CONTROL, int ROWS>
__device__ __forceinline__ double plus_before(double v) {
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, CONTROL, ROWS, 0xf, false);
  const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), CONTROL, ROWS, 0xf, false);
  return v + __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
__device__ __forceinline__ double wave_scan(double v) {
  v = plus_before<0x111, 0xf>(v);
  v = plus_before<0x112, 0xf>(v);
  v = plus_before<0x114, 0xf>(v);
  v = plus_before<0x118, 0xf>(v);
  v = plus_before<0x142, 0xa>(v);
  return plus_before<0x143, 0xc>(v);
}

// The sum over a workgroup, in every thread; `space` has room for a value per wavefront and may be used again behind the next barrier.
template <int THREADS = kVerThreads>
__device__ __forceinline__ double group_sum(double v, double* space) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) space[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) s += space[w];
  return s;
}

// Some chunks of one row: the parts of its softmax.  Grid: (`groups` workgroups to a row) x (1, or 2 with draft rows).  The next chunk is on its way while
// this one is summed.
template <typename T>
__global__ void __launch_bounds__(kVerThreads) verify_parts_kernel(const VerifyArgs a, int groups, const Divide by_groups) {
  __shared__ float tops[kVerThreads / 64];
  __shared__ int places[kVerThreads / 64];
  __shared__ double sums[kVerThreads / 64];
  __shared__ uint32_t table[2 * kVerTable];
  const int row = by_groups.of(blockIdx.x), b = row / a.nodes, node = row - b * a.nodes;
  const char* from = blockIdx.y == 0 ? a.logits + (b * a.logits_batch + node * a.logits_node) * (int64_t)sizeof(T)
                                     : a.draft + (b * a.draft_batch + node * a.draft_node) * (int64_t)sizeof(T);
  const float temperature = a.temperature[b];
  if (blockIdx.y == 1 && greedy(temperature)) return;
  int chunk = blockIdx.x - row * groups;
  typename Chunk<T>::Raw raw;
  raw.load(from, chunk, a.vocabulary);
  fill_table(table);
  const double by = 1.0 / (double)temperature;
  while (true) {
    Chunk<T> c;
    c.take(raw);
    const int next = chunk + groups;
    if (next < a.chunks) raw.load(from, next, a.vocabulary);
    float top = -INFINITY;
#pragma unroll
    for (int p = 0; p < kVerPieces; ++p)
#pragma unroll
      for (int e = 0; e < Chunk<T>::E; ++e) top = fmaxf(top, c.x[p][e]);
    top = wave_all(top, [](float x, float y) { return fmaxf(x, y); });
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kVerThreads / 64; ++w) top = fmaxf(top, tops[w]);
    VerifyPart part{0.0, top, 0x7fffffff};
    // (either way ends behind a second barrier, so the tops may be written again)
    if (greedy(temperature)) {
      int at = 0x7fffffff;
#pragma unroll
      for (int p = 0; p < kVerPieces; ++p)
#pragma unroll
        for (int e = 0; e < Chunk<T>::E; ++e)
          if (c.x[p][e] == top && top != -INFINITY) at = min(at, Chunk<T>::index(from, chunk, p, e));
      at = wave_all(at, [](int x, int y) { return min(x, y); });
      if ((threadIdx.x & 63) == 0) places[threadIdx.x >> 6] = at;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kVerThreads / 64; ++w) part.at = min(part.at, places[w]);
    } else {
      const Weigher w(table, top, by);
      double s = 0.0;
      if (w.plain) {
#pragma unroll
        for (int p = 0; p < kVerPieces; ++p)
#pragma unroll
          for (int e = 0; e < Chunk<T>::E; ++e) s = w.plus(c.x[p][e], s);
      } else {
        for (int i = threadIdx.x; i < Chunk<T>::kElements; i += kVerThreads) {
          const int at = chunk * Chunk<T>::kElements + i - Chunk<T>::lead(from);
          if (at >= 0 && at < a.vocabulary) s += weight(number(logit<T>(from, at)), top, by);
        }
      }
      part.sum = group_sum(s, sums);
    }
    if (threadIdx.x == 0) a.parts[((int64_t)blockIdx.y * a.batch * a.nodes + row) * a.chunks + chunk] = part;
    if (next >= a.chunks) return;
    chunk = next;
  }
}

// The softmax of a whole row from its parts, by one wavefront; every lane has the answer.  by: 1 / temperature; best: the best token is
// asked for, not the sum.
struct RowTop {
  float top;
  int at;          // greedy: the first place of the largest; 0x7fffffff: the row has no number
  double sum;
};
// mine: my_part(), which may be asked for long before.
__device__ __forceinline__ VerifyPart my_part(const VerifyPart* parts, int chunks) {
  const int lane = threadIdx.x & 63;
  return lane < chunks ? parts[lane] : VerifyPart{0.0, -INFINITY, 0x7fffffff};
}
__device__ __forceinline__ RowTop row_top(const VerifyPart* parts, int chunks, double by, bool best, const VerifyPart& mine) {
  RowTop r{-INFINITY, 0x7fffffff, 0.0};
  const int lane = threadIdx.x & 63;
  float top = mine.top;
  for (int i = lane + 64; i < chunks; i += 64) top = fmaxf(top, parts[i].top);
  r.top = wave_all(top, [](float x, float y) { return fmaxf(x, y); });
  if (best) {
    r.at = mine.top == r.top ? mine.at : 0x7fffffff;
    for (int i = lane + 64; i < chunks; i += 64)
      if (parts[i].top == r.top) r.at = min(r.at, parts[i].at);
    r.at = wave_all(r.at, [](int x, int y) { return min(x, y); });
  } else {
    r.sum = mine.sum * weight(mine.top, r.top, by);
    for (int i = lane + 64; i < chunks; i += 64) r.sum += parts[i].sum * weight(parts[i].top, r.top, by);
    r.sum = wave_sum(r.sum);
  }
  return r;
}

// max(p - a q, 0) of a word from its weights; with a > 0 scale_p has kSure in it.  Both products are rounded before they meet: one that is subtracted as it is from a
// rounded one leaves its rounding.  `none` is taken off besides.
__device__ __forceinline__ double left_of(double weight_p, double scale_p, double weight_q, double scale_q, double none) {
#pragma clang fp contract(off)
  const double p = weight_p * scale_p, q = __builtin_fma(weight_q, scale_q, none);
  return __builtin_fmax(p - q, 0.0);
}

// Weights and rows' sums are good to 1e-13 each, and two rows may be cut into chunks at different words: of a word of which less than 4e-13 of its probability is left
// beside the draft nothing may be left in truth, and nothing is taken to be, so that equal rows leave nothing at all.  What is left of others may be as little as it will.
constexpr double kNothingLeft = 4e-13, kSure = 1.0 - kNothingLeft;

// Chunks of less than this are not drawn from.  A word's weight counts from 1e-290 of the whole on where it is drawn, and a chunk of 8192 words that comes to 1e-280 has one.
constexpr double kLeastChunk = 1e-280;

// What the tests of a row's children came to.
struct RowState {
  int taken;        // the child that stands, or -1
  int level;        // -1: what is left is p; j: max(p - a q, 0) of sums rest[j]
  double a, sum;    // of that level
  bool open;        // the sum that the next test needs is not there yet
  int refused;      // children refused so far
};

struct RowInfo {
  RowTop p, q;
  RowState s;
};

// A sequence's tree, in LDS; a chain where no parents are given.  A barrier has to follow.
struct Tree {
  int parents[kVerMaxNodes], tokens[kVerMaxNodes];
};
__device__ __forceinline__ void load_tree(const VerifyArgs& g, int b, Tree& t) {
  for (int i = threadIdx.x; i < g.nodes; i += blockDim.x) {
    t.parents[i] = g.parents == nullptr ? i - 1 : g.parents[(int64_t)b * g.nodes + i];
    t.tokens[i] = g.tokens[(int64_t)b * g.nodes + i];
  }
}

// The child that a lane looks at: node `first` + lane, if it is one of `node`'s.
struct Child {
  bool is;
  int word;
  float u, x, y;      // its uniform and its logits
};
template <typename T>
__device__ __forceinline__ Child child_of(const VerifyArgs& g, const int32_t* parents, const int32_t* tokens, int b, int node, int first) {
  const int mine = first + (threadIdx.x & 63);
  Child c{mine < g.nodes && (parents == nullptr ? mine - 1 : parents[mine]) == node, -1, 0.f, -INFINITY, -INFINITY};
  if (c.is) {
    c.word = tokens[mine];
    c.u = g.uniforms[(int64_t)b * g.nodes + mine];
    if ((uint32_t)c.word < (uint32_t)g.vocabulary) {
      const char* from_p = g.logits + (b * g.logits_batch + node * g.logits_node) * (int64_t)sizeof(T);      // both on their way before either is looked at
      const char* from_q = g.draft == nullptr ? from_p : g.draft + (b * g.draft_batch + node * g.draft_node) * (int64_t)sizeof(T);
      const T x = reinterpret_cast<const T*>(from_p)[c.word], y = reinterpret_cast<const T*>(from_q)[c.word];
      c.x = number((float)x);
      c.y = number((float)y);
    }
  }
  return c;
}

// Tests the children of a node of a sequence with a temperature, by one wavefront; parents (nullptr: a chain) and tokens are the sequence's, c its
// child_of() from the node behind it on, which is asked for before the sums are known.  `ready` sums of max(p - a q, 0) are there.  Several kernels come to
// the same answers here, so nothing is left to how a compiler pairs products and sums.
template <typename T>
__device__ RowState test_children(const VerifyArgs& g, const int32_t* parents, const int32_t* tokens, int b, int node, int ready, const RowTop& p, const RowTop& q,
                                  Child c) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63, row = b * g.nodes + node;
  const double by = 1.0 / (double)g.temperature[b];
  auto parent = [&](int i) { return parents == nullptr ? i - 1 : parents[i]; };
  RowState s{-1, -1, 0.0, 1.0, false, 0};
  double gone = 0.0;      // without draft rows: the probability of the refused
  for (int first = node + 1; first < g.nodes; first += 64) {
    if (first > node + 1) c = child_of<T>(g, parents, tokens, b, node, first);
    const bool child = c.is;
    const int word = c.word;
    const double u = (double)c.u;
    // every lane forms the probabilities of its own node, then the children are gone through in order
    const double pw = child && p.sum > 0.0 ? weight(c.x, p.top, by) / p.sum : 0.0, qw = child && q.sum > 0.0 ? weight(c.y, q.top, by) / q.sum : 0.0;
    for (uint64_t left = __ballot(child); left != 0; left &= left - 1) {
      const int l = __ffsll((unsigned long long)left) - 1;
      const double cu = of_lane(u, l), cp = of_lane(pw, l), cq = of_lane(qw, l);
      if (g.draft == nullptr) {
        // a word that was refused before has left already
        const int w = __builtin_amdgcn_readlane(word, l);
        bool before = __any(child && lane < l && word == w);
        for (int i = node + 1; !before && i < first; i += 64)
          before = __any(i + lane < first && parent(i + lane) == node && tokens[i + lane] == w);
        const double have = before ? 0.0 : cp;
        if (cu * (1.0 - gone) < have) {
          s.taken = first + l;
          return s;
        }
        if (1.0 - gone - have > kNothingLeft) gone += have;
        ++s.refused;
        continue;
      }
      const double have = s.level < 0 ? cp : __builtin_fmax(cp * kSure - s.a * cq, 0.0) / s.sum;
      if (cu * cq < have) {
        s.taken = first + l;
        return s;
      }
      // refused: one more sum over the row
      const int j = s.refused;
      if (j >= g.siblings) return s;      // no room for more: the caller gave the most children a node has
      if (j >= ready) {
        s.open = true;
        return s;
      }
      ++s.refused;
      double rest = 0.0;
      for (int i = lane; i < g.chunks; i += 64) rest += g.rest[((int64_t)j * g.batch * g.nodes + row) * g.chunks + i];
      rest = wave_sum(rest);
      if (rest > 0.0) {      // (else nothing of the target is left beside the draft, and the distribution stays)
        s.a += s.sum;
        s.sum = rest;
        s.level = j;
      }
    }
  }
  return s;
}

// What `round` sums tell about every row; one row to a wavefront.
template <typename T>
__global__ void __launch_bounds__(kVerThreads) verify_rows_kernel(const VerifyArgs a, int round) {
  const int row = blockIdx.x * (kVerThreads / 64) + (threadIdx.x >> 6);
  if (row >= a.batch * a.nodes) return;
  const int b = row / a.nodes, node = row - b * a.nodes;
  const float temperature = a.temperature[b];
  if (greedy(temperature)) return;
  const double by = 1.0 / (double)temperature;
  const int32_t *parents = a.parents == nullptr ? nullptr : a.parents + (int64_t)b * a.nodes, *tokens = a.tokens + (int64_t)b * a.nodes;
  const VerifyPart *parts = a.parts + (int64_t)row * a.chunks, *draft_parts = parts + (int64_t)a.batch * a.nodes * a.chunks;
  VerifyPart part{}, draft_part{};
  if (round == 0) {
    part = my_part(parts, a.chunks);
    draft_part = my_part(draft_parts, a.chunks);
  }
  const Child child = child_of<T>(a, parents, tokens, b, node, node + 1);
  RowInfo info;
  if (round == 0) {
    info.p = row_top(parts, a.chunks, by, false, part);
    info.q = row_top(draft_parts, a.chunks, by, false, draft_part);
  } else {
    info = a.infos[row];
  }
  info.s = test_children<T>(a, parents, tokens, b, node, round, info.p, info.q, child);
  if ((threadIdx.x & 63) == 0) a.infos[row] = info;
}

// Some chunks of a row whose children were refused up to round `round`: the sums of max(p - a q, 0) with the next a.  Grid: `groups` workgroups to a row.
// A row that the path does not come to is not worth the sum: some ancestor has taken another child, or none.
template <typename T>
__global__ void __launch_bounds__(kVerThreads) verify_rest_kernel(const VerifyArgs a, int round, int groups) {
  __shared__ double sums[kVerThreads / 64];
  __shared__ uint32_t table[2 * kVerTable];
  __shared__ int parents[kVerMaxNodes], taken[kVerMaxNodes], wanted;      // taken: -2 where it is still open
  const int row = blockIdx.x / groups, b = row / a.nodes, node = row - b * a.nodes;
  const float temperature = a.temperature[b];
  if (greedy(temperature)) return;
  const RowInfo info = a.infos[row];
  if (!info.s.open) return;
  for (int i = threadIdx.x; i < a.nodes; i += kVerThreads) {
    const RowState& s = a.infos[(int64_t)b * a.nodes + i].s;
    parents[i] = a.parents == nullptr ? i - 1 : a.parents[(int64_t)b * a.nodes + i];
    taken[i] = s.open ? -2 : s.taken;
  }
  fill_table(table);
  __syncthreads();
  if (threadIdx.x == 0) {
    int at = node;
    bool comes = true;
    while (comes && at > 0) {
      const int up = parents[at];
      comes = (uint32_t)up < (uint32_t)at && (taken[up] == at || taken[up] == -2);
      at = up;
    }
    wanted = comes;
  }
  __syncthreads();
  if (!wanted) return;
  const RowTop p = info.p, q = info.q;
  const double by = 1.0 / (double)temperature, next_a = info.s.a + info.s.sum;
  const char* from_p = a.logits + (b * a.logits_batch + node * a.logits_node) * (int64_t)sizeof(T);
  const char* from_q = a.draft + (b * a.draft_batch + node * a.draft_node) * (int64_t)sizeof(T);
  const double scale_p = p.sum > 0.0 ? kSure / p.sum : 0.0, scale_q = q.sum > 0.0 ? next_a / q.sum : 0.0;
  const Weigher wp(table, p.top, by), wq(table, q.top, by);
  const bool plain = wp.plain && wq.plain, alike = Chunk<T>::lead(from_p) == Chunk<T>::lead(from_q);
  for (int chunk = blockIdx.x - row * groups; chunk < a.chunks; chunk += groups) {
    Chunk<T> c, d;
    c.load(from_p, chunk, a.vocabulary);
    if (alike) {
      d.load(from_q, chunk, a.vocabulary);
    } else {
#pragma unroll
      for (int i = 0; i < kVerPieces; ++i)
#pragma unroll
        for (int e = 0; e < Chunk<T>::E; ++e) {
          const int at = Chunk<T>::index(from_p, chunk, i, e);
          d.x[i][e] = at >= 0 && at < a.vocabulary ? number(logit<T>(from_q, at)) : -INFINITY;
        }
    }
    double s = 0.0;
    if (plain) {      // (1e-290 is above what a word without a probability has here and nothing beside one that has any)
#pragma unroll
      for (int i = 0; i < kVerPieces; ++i)
#pragma unroll
        for (int e = 0; e < Chunk<T>::E; ++e) s += left_of(wp.of(c.x[i][e]), scale_p, wq.of(d.x[i][e]), scale_q, 1e-290);
    } else {
#pragma unroll
      for (int i = 0; i < kVerPieces; ++i)
#pragma unroll 1
        for (int e = 0; e < Chunk<T>::E; ++e) {
          float x = c.x[i][0], y = d.x[i][0];
#pragma unroll
          for (int j = 1; j < Chunk<T>::E; ++j) {
            x = e == j ? c.x[i][j] : x;
            y = e == j ? d.x[i][j] : y;
          }
          s += left_of(weight(number(x), p.top, by), scale_p, weight(number(y), q.top, by), scale_q, 0.0);
        }
    }
    __syncthreads();
    s = group_sum(s, sums);
    if (threadIdx.x == 0) a.rest[((int64_t)round * a.batch * a.nodes + row) * a.chunks + chunk] = s;
  }
}

constexpr int kVerChooseThreads = kVerThreads * kVerPieces;      // one piece of a chunk to a thread

// One sequence: which child of every node stands, the path from the root along them, and the token behind it: the first word whose running sum of what is
// left of the last node's distribution exceeds uniforms[0] times the whole.  The nodes are tested side by side, one to a wavefront, and what is found out about them
// is kept for the one that turns out to be the last.
template <typename T>
__global__ void __launch_bounds__(kVerChooseThreads) verify_choose_kernel(const VerifyArgs a) {
  constexpr int WAVES = kVerChooseThreads / 64, E = Chunk<T>::E;
  __shared__ Tree tree;
  __shared__ RowState states[kVerMaxNodes];
  __shared__ RowTop tops[kVerMaxNodes], draft_tops[kVerMaxNodes];
  __shared__ double sums[WAVES], before_chunk, gone_weights[kVerMaxNodes];
  __shared__ uint32_t table[2 * kVerTable];
  __shared__ int end, length, the_chunk, gone_count, found[WAVES], lasts[WAVES], gone[kVerMaxNodes];
  const int b = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const float temperature = a.temperature[b];
  const bool best = greedy(temperature), named = a.draft == nullptr;
  const double by = best ? 0.0 : 1.0 / (double)temperature;
  const int64_t rows = (int64_t)a.batch * a.nodes;
  load_tree(a, b, tree);
  fill_table(table);
  __syncthreads();
  for (int node = wave; node < a.nodes; node += WAVES) {
    RowTop p, q{};
    Child child{};
    const VerifyPart* parts = a.parts + (b * a.nodes + node) * (int64_t)a.chunks;
    VerifyPart part{};
    if (best || named) part = my_part(parts, a.chunks);
    if (!best) child = child_of<T>(a, tree.parents, tree.tokens, b, node, node + 1);
    if (best || named) {
      p = row_top(parts, a.chunks, by, best, part);
    } else {
      p = a.infos[b * a.nodes + node].p;
      q = a.infos[b * a.nodes + node].q;
    }
    RowState s{-1, -1, 0.0, 1.0, false, 0};
    if (best) {
      for (int first = node + 1; first < a.nodes && s.taken < 0; first += 64) {
        const int mine = first + lane;
        const uint64_t same = __ballot(mine < a.nodes && p.at != 0x7fffffff && tree.parents[mine] == node && tree.tokens[mine] == p.at);
        if (same != 0) s.taken = first + __ffsll((unsigned long long)same) - 1;
      }
    } else {
      s = test_children<T>(a, tree.parents, tree.tokens, b, node, a.siblings, p, q, child);
    }
    if (lane == 0) {
      tops[node] = p;
      draft_tops[node] = q;
      states[node] = s;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    int node = 0, n = 0;
    while (states[node].taken >= 0) {      // children have higher numbers than their parents, so this ends
      a.path[(int64_t)b * a.nodes + n] = node;
      node = states[node].taken;
      a.words[(int64_t)b * a.nodes + n] = tree.tokens[node];
      ++n;
    }
    a.path[(int64_t)b * a.nodes + n] = node;
    end = node;
    length = n;
    a.count[b] = n + 1;
  }
  __syncthreads();
  const int node = end;
  for (int i = length + 1 + threadIdx.x; i < a.nodes; i += kVerChooseThreads) {
    a.path[(int64_t)b * a.nodes + i] = -1;
    a.words[(int64_t)b * a.nodes + i] = -1;
  }
  int32_t* out = a.words + (int64_t)b * a.nodes + length;
  const RowTop p = tops[node], q = draft_tops[node];
  const RowState s = states[node];
  if (best || !(p.sum > 0.0)) {
    if (threadIdx.x == 0) *out = best && p.at != 0x7fffffff ? p.at : -1;
    return;
  }
  const char* from_p = a.logits + (b * a.logits_batch + node * a.logits_node) * (int64_t)sizeof(T);
  const char* from_q = named ? nullptr : a.draft + (b * a.draft_batch + node * a.draft_node) * (int64_t)sizeof(T);
  const int64_t row = (int64_t)b * a.nodes + node;
  const int lead = Chunk<T>::lead(from_p);
  if (wave == 0) {
    // without draft rows: the words that were refused and are gone.  A word that is named twice goes once, and one that is all there is stays.
    int n = 0;
    double left = 1.0;
    for (int first = node + 1; named && first < a.nodes; first += 64) {
      const int mine = first + lane;
      const bool child = mine < a.nodes && tree.parents[mine] == node && (uint32_t)tree.tokens[mine] < (uint32_t)a.vocabulary;
      const int word = child ? tree.tokens[mine] : -1;
      const double have = child ? weight(number(logit<T>(from_p, word)), p.top, by) / p.sum : 0.0;
      for (uint64_t rest = __ballot(child); rest != 0; rest &= rest - 1) {
        const int l = __ffsll((unsigned long long)rest) - 1, w = __builtin_amdgcn_readlane(word, l);
        const double pw = of_lane(have, l);
        bool before = false;
        for (int i = lane; i < n; i += 64) before = before || gone[i] == w;
        if (__any(before) || !(left - pw > kNothingLeft)) continue;
        left -= pw;
        if (lane == 0) {
          gone[n] = w;
          gone_weights[n] = pw;
        }
        ++n;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }
    // The weight of a chunk in what is left.  A sum less its refused parts is off by 1e-13 of them at most (Weigher; those that are the largest of their chunk are
    // exact).  Where a share s of the whole is left, and the chance that it comes to that is s, this is 1e-13 / s of it: one draw in 10^13 goes elsewhere.  A chunk in
    // which that is all there is has nothing to draw.
    auto chunk_weight = [&](int i) {
      if (s.level >= 0) {
        const double w = a.rest[(s.level * rows + row) * a.chunks + i];
        return w > kLeastChunk ? w : 0.0;
      }
      const VerifyPart part = a.parts[row * a.chunks + i];
      double w = part.sum * weight(part.top, p.top, by) / p.sum, refused = 0.0;
      for (int j = 0; j < n; ++j)
        if ((gone[j] + lead) / Chunk<T>::kElements == i) refused += gone_weights[j];
      w -= refused;
      return w > 2e-13 * refused && w > kLeastChunk ? w : 0.0;
    };
    const double first_weight = lane < a.chunks ? chunk_weight(lane) : 0.0;
    double whole = first_weight;
    for (int i = lane + 64; i < a.chunks; i += 64) whole += chunk_weight(i);
    whole = wave_sum(whole);
    const double at = (double)a.uniforms[(int64_t)b * a.nodes] * whole;
    double before = 0.0, chosen_before = 0.0, with_before = 0.0;
    int chosen = -1, with = -1;
    for (int first = 0; first < a.chunks && chosen < 0; first += 64) {
      const double w = first == 0 ? first_weight : first + lane < a.chunks ? chunk_weight(first + lane) : 0.0;
      const double run = wave_scan(w) + before;
      const uint64_t over = __ballot(run > at && w > 0.0), some = __ballot(w > 0.0);
      if (over != 0) {
        const int l = __ffsll((unsigned long long)over) - 1;
        chosen = first + l;
        chosen_before = __shfl(run - w, l);
      }
      if (some != 0) {
        const int l = 63 - __clzll((unsigned long long)some);
        with = first + l;
        with_before = __shfl(run - w, l);
      }
      before = __shfl(run, 63);
    }
    if (chosen < 0) {      // a uniform of 1 or more: the last that has a weight
      chosen = with;
      chosen_before = with_before;
    }
    if (lane == 0) {
      the_chunk = chosen;
      before_chunk = at - chosen_before;
      gone_count = n;
    }
  }
  __syncthreads();
  const int chunk = the_chunk, goners = gone_count;
  if (chunk < 0) {
    if (threadIdx.x == 0) *out = -1;
    return;
  }
  // inside the chunk: a piece to a thread, in the order of the row
  const double scale_p = (s.level >= 0 ? kSure : 1.0) / p.sum, scale_q = !named && q.sum > 0.0 ? s.a / q.sum : 0.0, need = before_chunk;
  const int start = chunk * Chunk<T>::kElements + (int)threadIdx.x * E - lead;
  auto piece = [&](const char* from, bool even) {
    typename Piece<T>::type v;
    if (even && start >= 0 && start + E <= a.vocabulary) {
      v = *reinterpret_cast<const typename Piece<T>::type*>(from + (int64_t)start * sizeof(T));
    } else {      // all on their way at once: places outside the row read its ends
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = reinterpret_cast<const T*>(from)[min(max(start + e, 0), a.vocabulary - 1)];
    }
    return v;
  };
  const typename Piece<T>::type of_p = piece(from_p, true);
  typename Piece<T>::type of_q{};
  if (scale_q != 0.0) of_q = piece(from_q, Chunk<T>::lead(from_q) == lead);
  float x[E], y[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    x[e] = start + e >= 0 && start + e < a.vocabulary ? number((float)of_p[e]) : -INFINITY;
    y[e] = number((float)of_q[e]);
  }
  const Weigher wp(table, p.top, by), wq(table, q.top, by);
  double w[E], mine = 0.0;
  if (wp.plain && (scale_q == 0.0 || wq.plain)) {      // (1e-290 as in the sums of what is left)
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = left_of(wp.of(x[e]), scale_p, scale_q != 0.0 ? wq.of(y[e]) : 0.0, scale_q, 1e-290);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = left_of(weight(x[e], p.top, by), scale_p, scale_q != 0.0 ? weight(y[e], q.top, by) : 0.0, scale_q, 0.0);
  }
  for (int j = 0; j < goners; ++j)
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = gone[j] == start + e ? 0.0 : w[e];
#pragma unroll
  for (int e = 0; e < E; ++e) mine += w[e];
  const double upto = wave_scan(mine);
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  double at = upto - mine;
#pragma unroll
  for (int i = 0; i < WAVES - 1; ++i) at += i < wave ? sums[i] : 0.0;
  int answer = 0x7fffffff, last = -1;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    at += w[e];
    if (w[e] > 0.0) {
      if (at > need) answer = min(answer, start + e);
      last = start + e;
    }
  }
  answer = wave_all(answer, [](int x, int y) { return min(x, y); });
  last = wave_all(last, [](int x, int y) { return max(x, y); });
  if (lane == 0) {
    found[wave] = answer;
    lasts[wave] = last;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      answer = min(answer, found[i]);
      last = max(last, lasts[i]);
    }
    *out = answer != 0x7fffffff ? answer : last;
  }
}

}  // namespace dpllm
