// Verification of drafted tokens.  p_i = softmax(logits_i / temperature) and q_i = softmax(draft_i / temperature) of node i.  The children c of a node, in the
// order of their numbers, are taken with probability min(1, r(c) / q(c)), r = p at first, and r <- max(r - q, 0) / (its sum) behind a child that was
// not.  All those r have one form: r_j = max(p - a_j q, 0) / S_j, a_0 = 0, S_0 = 1, a_(j+1) = a_j + S_j, S_j = sum of max(p - a_j q, 0) (with
// r_j = max(p - a_j q, 0) / S_j, r_j - q is (p - a_j q - S_j q) / S_j where that is positive), so a row's state is two numbers and one more
// sum over the row moves it on.  Without draft rows a child was named, not drawn, and leaves the distribution when it is not taken.
//
// Answers are whole numbers, so nothing may hang on the order of additions: logits are widened, and differences, exponentials and sums are kept, in
// 64 bits; two orders of a sum of 10^5 terms differ by about 1e-14, and so do the numbers that a probability of 2^-24 steps is compared with.
#pragma once
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

struct VerifyArgs {
  const char *logits, *draft;
  int64_t logits_batch, logits_node, draft_batch, draft_node;      // elements
  const int32_t *tokens, *parents;
  const float *uniforms, *temperature;
  int32_t *count, *path, *words;
  VerifyPart* parts;       // [2 with draft rows][batch * nodes][chunks]
  double* rest;            // [siblings][batch * nodes][chunks]: sums of max(p - a q, 0)
  int batch, nodes, vocabulary, chunks, siblings;
  Divide by_chunks;
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

// The temperature of a sequence: 0 (or less, or NaN) takes the best token.
__device__ __forceinline__ bool greedy(float temperature) { return !(temperature > 0.f); }

template <typename T>
__device__ __forceinline__ float logit(const char* row, int i) { return (float)reinterpret_cast<const T*>(row)[i]; }

// A chunk of a row in registers: piece p of a thread is the 16 bytes (p * threads + thread) of the chunk, counted from the last 16-byte boundary in front
// of the row.  Pieces that the row covers in part are read element by element; what lies outside, and NaN, is -infinity.
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
  __device__ __forceinline__ void load(const char* row, int chunk, int n) {
    const T* base = reinterpret_cast<const T*>(row);
#pragma unroll
    for (int p = 0; p < kVerPieces; ++p) {
      const int i = index(row, chunk, p, 0);
      if (i >= 0 && i + E <= n) {
        const typename Piece<T>::type v = *reinterpret_cast<const typename Piece<T>::type*>(base + i);
#pragma unroll
        for (int e = 0; e < E; ++e) x[p][e] = (float)v[e];
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[p][e] = i + e >= 0 && i + e < n ? (float)base[i + e] : -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) x[p][e] = x[p][e] == x[p][e] ? x[p][e] : -INFINITY;
    }
  }
};

template <typename T, typename F>
__device__ __forceinline__ T wave_all(T v, F f) {
#pragma unroll
  for (int i = 1; i < 64; i *= 2) v = f(v, __shfl_xor(v, i));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
  return wave_all(v, [](double a, double b) { return a + b; });
}

// The sum over a workgroup, in every thread; `space` has room for a value per wavefront and may be used again behind the next barrier.
__device__ __forceinline__ double group_sum(double v, double* space) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) space[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kVerThreads / 64; ++w) s += space[w];
  return s;
}

// One chunk of one row: the parts of its softmax.  Grid: (chunks x rows) x (1, or 2 with draft rows).
template <typename T>
__global__ void __launch_bounds__(kVerThreads) verify_parts_kernel(const VerifyArgs a) {
  __shared__ float tops[kVerThreads / 64];
  __shared__ int places[kVerThreads / 64];
  __shared__ double sums[kVerThreads / 64];
  const int row = a.by_chunks.of(blockIdx.x), chunk = blockIdx.x - row * a.chunks, b = row / a.nodes, node = row - b * a.nodes;
  const char* from = blockIdx.y == 0 ? a.logits + (b * a.logits_batch + node * a.logits_node) * (int64_t)sizeof(T)
                                     : a.draft + (b * a.draft_batch + node * a.draft_node) * (int64_t)sizeof(T);
  const float temperature = a.temperature[b];
  if (blockIdx.y == 1 && greedy(temperature)) return;
  Chunk<T> c;
  c.load(from, chunk, a.vocabulary);
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
    const double by = 1.0 / (double)temperature;
    double s = 0.0;
#pragma unroll
    for (int p = 0; p < kVerPieces; ++p)
#pragma unroll
      for (int e = 0; e < Chunk<T>::E; ++e) s += weight(c.x[p][e], top, by);
    part.sum = group_sum(s, sums);
  }
  if (threadIdx.x == 0) a.parts[((int64_t)blockIdx.y * a.batch * a.nodes + row) * a.chunks + chunk] = part;
}

// The softmax of a whole row from its parts, by one wavefront; every lane has the answer.
struct RowTop {
  float top;
  int at;          // greedy: the first place of the largest; 0x7fffffff: the row has no number
  double sum;
};
__device__ __forceinline__ RowTop row_top(const VerifyPart* parts, int chunks, double by) {
  RowTop r{-INFINITY, 0x7fffffff, 0.0};
  const int lane = threadIdx.x & 63;
  float top = -INFINITY;
  for (int i = lane; i < chunks; i += 64) top = fmaxf(top, parts[i].top);
  r.top = wave_all(top, [](float x, float y) { return fmaxf(x, y); });
  for (int i = lane; i < chunks; i += 64) {
    if (parts[i].top == r.top) r.at = min(r.at, parts[i].at);
    r.sum += parts[i].sum * weight(parts[i].top, r.top, by);
  }
  r.at = wave_all(r.at, [](int x, int y) { return min(x, y); });
  r.sum = wave_sum(r.sum);
  return r;
}

// What the tests of a row's children came to.
struct RowState {
  int taken;        // the child that stands, or -1
  int level;        // -1: what is left is p; j: max(p - a q, 0) of sums rest[j]
  double a, sum;    // of that level
  bool open;        // the sum that the next test needs is not there yet
  int refused;      // children refused so far
};

// The parent of a node; a chain where no parents are given.
__device__ __forceinline__ int parent_of(const VerifyArgs& g, int b, int node) {
  return g.parents == nullptr ? node - 1 : g.parents[(int64_t)b * g.nodes + node];
}

// Tests the children of a node of a sequence with a temperature, by one wavefront.  `ready` sums of max(p - a q, 0) are there.  Several kernels come to
// the same answers here, so nothing is left to how a compiler pairs products and sums.
template <typename T>
__device__ RowState test_children(const VerifyArgs& g, int b, int node, int ready, const RowTop& p, const RowTop& q) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63, row = b * g.nodes + node;
  const char* from_p = g.logits + (b * g.logits_batch + node * g.logits_node) * (int64_t)sizeof(T);
  const char* from_q = g.draft == nullptr ? nullptr : g.draft + (b * g.draft_batch + node * g.draft_node) * (int64_t)sizeof(T);
  const double by = 1.0 / (double)g.temperature[b];
  RowState s{-1, -1, 0.0, 1.0, false, 0};
  double gone = 0.0;      // without draft rows: the probability of the refused
  for (int first = node + 1; first < g.nodes; first += 64) {
    const int mine = first + lane;
    const bool child = mine < g.nodes && parent_of(g, b, mine) == node;
    // every lane forms the probabilities of its own node, then the children are gone through in order
    int word = -1;
    double u = 0.0, pw = 0.0, qw = 0.0;
    if (child) {
      word = g.tokens[(int64_t)b * g.nodes + mine];
      u = (double)g.uniforms[(int64_t)b * g.nodes + mine];
      if ((uint32_t)word < (uint32_t)g.vocabulary) {
        const float x = logit<T>(from_p, word);
        pw = p.sum > 0.0 ? weight(x == x ? x : -INFINITY, p.top, by) / p.sum : 0.0;
        if (from_q != nullptr) {
          const float y = logit<T>(from_q, word);
          qw = q.sum > 0.0 ? weight(y == y ? y : -INFINITY, q.top, by) / q.sum : 0.0;
        }
      }
    }
    for (uint64_t left = __ballot(child); left != 0; left &= left - 1) {
      const int l = __ffsll((unsigned long long)left) - 1;
      const double cu = __shfl(u, l), cp = __shfl(pw, l), cq = __shfl(qw, l);
      if (from_q == nullptr) {
        // a word that was refused before has left already
        const int w = __shfl(word, l);
        bool before = __any(child && lane < l && word == w);
        for (int i = node + 1; !before && i < first; i += 64)
          before = __any(i + lane < first && parent_of(g, b, i + lane) == node && g.tokens[(int64_t)b * g.nodes + i + lane] == w);
        const double have = before ? 0.0 : cp;
        if (cu * (1.0 - gone) < have) {
          s.taken = first + l;
          return s;
        }
        if (1.0 - gone - have > 0.0) gone += have;
        ++s.refused;
        continue;
      }
      const double have = __builtin_fmax(cp - s.a * cq, 0.0);
      if (cu * cq * s.sum < have) {
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

// One chunk of a row whose children were refused up to round `round`: the sum of max(p - a q, 0) with the next a.  Grid: chunks x rows in one.
template <typename T>
__global__ void __launch_bounds__(kVerThreads) verify_rest_kernel(const VerifyArgs a, int round) {
  __shared__ double sums[kVerThreads / 64];
  __shared__ double shared_a[5];
  __shared__ int open;
  const int row = a.by_chunks.of(blockIdx.x), chunk = blockIdx.x - row * a.chunks, b = row / a.nodes, node = row - b * a.nodes;
  const float temperature = a.temperature[b];
  if (greedy(temperature)) return;
  const double by = 1.0 / (double)temperature;
  if (threadIdx.x < 64) {
    const RowTop p = row_top(a.parts + (int64_t)row * a.chunks, a.chunks, by);
    const RowTop q = row_top(a.parts + ((int64_t)a.batch * a.nodes + row) * a.chunks, a.chunks, by);
    const RowState s = test_children<T>(a, b, node, round, p, q);
    if (threadIdx.x == 0) {
      open = s.open;
      shared_a[0] = s.a + s.sum;
      shared_a[1] = p.sum;
      shared_a[2] = q.sum;
      shared_a[3] = p.top;
      shared_a[4] = q.top;
    }
  }
  __syncthreads();
  if (!open) return;
  const double next = shared_a[0], sum_p = shared_a[1], sum_q = shared_a[2];
  const float top_p = (float)shared_a[3], top_q = (float)shared_a[4];
  const char* from_p = a.logits + (b * a.logits_batch + node * a.logits_node) * (int64_t)sizeof(T);
  const char* from_q = a.draft + (b * a.draft_batch + node * a.draft_node) * (int64_t)sizeof(T);
  double s = 0.0;
  if (sum_p > 0.0) {
    const double scale_p = 1.0 / sum_p, scale_q = sum_q > 0.0 ? next / sum_q : 0.0;
    Chunk<T> c;
    c.load(from_p, chunk, a.vocabulary);
#pragma unroll
    for (int p = 0; p < kVerPieces; ++p)
#pragma unroll
      for (int e = 0; e < Chunk<T>::E; ++e) {
        const int i = Chunk<T>::index(from_p, chunk, p, e);
        if (c.x[p][e] == -INFINITY) continue;
        const float y = logit<T>(from_q, i);
        s += __builtin_fmax(weight(c.x[p][e], top_p, by) * scale_p - weight(y == y ? y : -INFINITY, top_q, by) * scale_q, 0.0);
      }
  }
  s = group_sum(s, sums);
  if (threadIdx.x == 0) a.rest[((int64_t)round * a.batch * a.nodes + row) * a.chunks + chunk] = s;
}

// One sequence: which child of every node stands, the path from the root along them, and the token behind it: the first word whose running sum of what is
// left of the last node's distribution exceeds uniforms[0] times the whole.
template <typename T>
__global__ void __launch_bounds__(kVerThreads) verify_choose_kernel(const VerifyArgs a) {
  __shared__ int taken[kVerMaxNodes];
  __shared__ RowState last_state;
  __shared__ RowTop last_p, last_q;
  __shared__ double sums[kVerThreads / 64], before_chunk;
  __shared__ int end, the_chunk, found[kVerThreads / 64];
  const int b = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const float temperature = a.temperature[b];
  const bool best = greedy(temperature);
  const double by = best ? 0.0 : 1.0 / (double)temperature;
  const int64_t rows = (int64_t)a.batch * a.nodes;
  auto top_of = [&](int node, int which) { return row_top(a.parts + (which * rows + b * a.nodes + node) * a.chunks, a.chunks, by); };
  for (int node = wave; node < a.nodes; node += kVerThreads / 64) {
    const RowTop p = top_of(node, 0);
    int t = -1;
    if (best) {
      for (int first = node + 1; first < a.nodes && t < 0; first += 64) {
        const int mine = first + lane;
        const uint64_t same = __ballot(mine < a.nodes && p.at != 0x7fffffff && parent_of(a, b, mine) == node && a.tokens[(int64_t)b * a.nodes + mine] == p.at);
        if (same != 0) t = first + __ffsll((unsigned long long)same) - 1;
      }
    } else {
      RowTop q{};
      if (a.draft != nullptr) q = top_of(node, 1);
      t = test_children<T>(a, b, node, a.siblings, p, q).taken;
    }
    if (lane == 0) taken[node] = t;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    int node = 0, n = 0;
    while (true) {      // children have higher numbers than their parents, so this ends
      a.path[(int64_t)b * a.nodes + n] = node;
      if (taken[node] < 0) break;
      node = taken[node];
      a.words[(int64_t)b * a.nodes + n] = a.tokens[(int64_t)b * a.nodes + node];
      ++n;
    }
    end = node;
    a.count[b] = n + 1;
    for (int i = n + 1; i < a.nodes; ++i) {
      a.path[(int64_t)b * a.nodes + i] = -1;
      a.words[(int64_t)b * a.nodes + i] = -1;
    }
    the_chunk = n;
  }
  __syncthreads();
  const int node = end;
  int32_t* out = a.words + (int64_t)b * a.nodes + the_chunk;
  __syncthreads();
  if (wave == 0) {
    const RowTop p = top_of(node, 0);
    RowTop q{};
    RowState s{-1, -1, 0.0, 1.0, false, 0};
    if (!best) {
      if (a.draft != nullptr) q = top_of(node, 1);
      s = test_children<T>(a, b, node, a.siblings, p, q);
    }
    if (lane == 0) {
      last_p = p;
      last_q = q;
      last_state = s;
    }
  }
  __syncthreads();
  const RowTop p = last_p, q = last_q;
  const RowState s = last_state;
  if (best || !(p.sum > 0.0)) {
    if (threadIdx.x == 0) *out = best && p.at != 0x7fffffff ? p.at : -1;
    return;
  }
  // without draft rows: the words that were refused and are gone.  A child's number is kept; the words are few.
  const bool named = a.draft == nullptr;
  const char* from_p = a.logits + (b * a.logits_batch + node * a.logits_node) * (int64_t)sizeof(T);
  const char* from_q = named ? nullptr : a.draft + (b * a.draft_batch + node * a.draft_node) * (int64_t)sizeof(T);
  int* gone = taken;      // the children of the last node, in order
  __shared__ int gone_count;
  if (threadIdx.x == 0) {
    int n = 0;
    if (named) {
      double left = 1.0;
      for (int i = node + 1; i < a.nodes; ++i) {
        if (parent_of(a, b, i) != node) continue;
        const int w = a.tokens[(int64_t)b * a.nodes + i];
        bool is_new = (uint32_t)w < (uint32_t)a.vocabulary;
        for (int j = 0; j < n; ++j) is_new = is_new && gone[j] != w;
        if (!is_new) continue;
        const float x = logit<T>(from_p, w);
        const double pw = weight(x == x ? x : -INFINITY, p.top, by) / p.sum;
        if (left - pw > 0.0) {
          left -= pw;
          gone[n++] = w;
        }
      }
    }
    gone_count = n;
  }
  __syncthreads();
  const int goners = gone_count;
  const int64_t row = (int64_t)b * a.nodes + node;
  const int lead = Chunk<T>::lead(from_p);
  // the weight of a chunk in what is left
  auto chunk_weight = [&](int i) {
    if (s.level >= 0) return a.rest[(s.level * rows + row) * a.chunks + i];
    const VerifyPart part = a.parts[row * a.chunks + i];
    double w = part.sum * weight(part.top, p.top, by) / p.sum;
    for (int j = 0; j < goners; ++j)
      if ((gone[j] + lead) / Chunk<T>::kElements == i) {
        const float x = logit<T>(from_p, gone[j]);
        w -= weight(x == x ? x : -INFINITY, p.top, by) / p.sum;
      }
    return __builtin_fmax(w, 0.0);
  };
  if (wave == 0) {
    double whole = 0.0;
    for (int i = lane; i < a.chunks; i += 64) whole += chunk_weight(i);
    whole = wave_sum(whole);
    const double at = (double)a.uniforms[(int64_t)b * a.nodes] * whole;
    double before = 0.0, chosen_before = 0.0;
    int chosen = -1, with = -1;
    double with_before = 0.0;
    for (int first = 0; first < a.chunks && chosen < 0; first += 64) {
      const double w = first + lane < a.chunks ? chunk_weight(first + lane) : 0.0;
      double run = w;
#pragma unroll
      for (int i = 1; i < 64; i *= 2) {
        const double v = __shfl_up(run, i);
        if (lane >= i) run += v;
      }
      run += before;
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
    }
  }
  __syncthreads();
  const int chunk = the_chunk;
  if (chunk < 0) {
    if (threadIdx.x == 0) *out = -1;
    return;
  }
  // inside the chunk: pieces in the order of the row are pieces in turn, then threads, then elements
  Chunk<T> c;
  c.load(from_p, chunk, a.vocabulary);
  const double scale_p = 1.0 / p.sum, scale_q = !named && q.sum > 0.0 ? s.a / q.sum : 0.0, need = before_chunk;
  double run = 0.0;
  int answer = 0x7fffffff, last = -1;
#pragma unroll
  for (int piece = 0; piece < kVerPieces; ++piece) {
    double w[Chunk<T>::E], mine = 0.0;
#pragma unroll
    for (int e = 0; e < Chunk<T>::E; ++e) {
      const int i = Chunk<T>::index(from_p, chunk, piece, e);
      w[e] = 0.0;
      if (c.x[piece][e] == -INFINITY) continue;
      w[e] = weight(c.x[piece][e], p.top, by) * scale_p;
      if (scale_q != 0.0) {
        const float y = logit<T>(from_q, i);
        w[e] = __builtin_fmax(w[e] - weight(y == y ? y : -INFINITY, q.top, by) * scale_q, 0.0);
      }
      for (int j = 0; j < goners; ++j)
        if (gone[j] == i) w[e] = 0.0;
    }
#pragma unroll
    for (int e = 0; e < Chunk<T>::E; ++e) mine += w[e];
    double upto = mine;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
      const double v = __shfl_up(upto, i);
      if (lane >= i) upto += v;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    double all = 0.0, front = 0.0;
#pragma unroll
    for (int i = 0; i < kVerThreads / 64; ++i) {
      if (i < wave) front += sums[i];
      all += sums[i];
    }
    double at = run + front + upto - mine;
#pragma unroll
    for (int e = 0; e < Chunk<T>::E; ++e) {
      at += w[e];
      if (w[e] > 0.0) {
        const int i = Chunk<T>::index(from_p, chunk, piece, e);
        if (at > need) answer = min(answer, i);
        last = max(last, i);
      }
    }
    run += all;
  }
  answer = wave_all(answer, [](int x, int y) { return min(x, y); });
  last = wave_all(last, [](int x, int y) { return max(x, y); });
  __syncthreads();
  if (lane == 0) found[wave] = answer;
  if (lane == 0) taken[wave] = last;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 0; i < kVerThreads / 64; ++i) {
      answer = min(answer, found[i]);
      last = max(last, taken[i]);
    }
    *out = answer != 0x7fffffff ? answer : last;
  }
}

}  // namespace dpllm
