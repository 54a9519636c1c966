// Attention of a few drafted tokens (the nodes of a tree) over a paged cache and over one another.
//
// For the row (node i, query head h) of a sequence: x_t = scale q . k_t over the tokens t of the cache and those nodes that the
// mask of i names, out = sum_t exp(x_t - m) v_t / sum_t exp(x_t - m), m the largest x_t; a row that sees nothing is zero.
#pragma once
#include "token_common.hpp"

namespace dpllm {

constexpr int kAttWaves = 4;        // wavefronts of a workgroup of the kernel for few rows, where the work is split
constexpr int kAttTile = 32;        // tokens of a step

struct AttentionArgs {
  CacheView cache;                  // of the layer
  Heads q, k_new, v_new, out;
  const int32_t* lens;
  const uint64_t* mask;             // [nodes][words]; nullptr: a chain
  int64_t mask_stride;
  float* lse;
  float* part;                      // [workgroups][rows of a tile][head_dim] where a sequence has several parts, then the tops and sums of the rows,
  float2* stats;                    // and where the parts of every sequence are
  int2* places;
  float scale, scale_log2;          // |scale|, and that / ln 2
  uint32_t sign, keep;              // sign: 0x80008000 for a negative scale, with which the queries change theirs; keep: 0 for a scale of 0, of which they are zeros
  Divide by_group;
  int batch, nodes, seen_nodes, words, kv_heads, group, rows, row_tiles, slots, least;      // least: steps of the smallest part worth a workgroup
};

template <typename T>
struct Matrix;
template <>
struct Matrix<half_t> {
  static constexpr uint32_t kNoNumber = 0x7c00u;   // the exponent of infinities and NaN
  // weights reach the matrix pipe as 2^12 times what they are (kLimit keeps them below the largest half), and are rounded to multiples of 2^-24, as a
  // half below 2^-14 is, only where they are below 2^-26 of the top's
  static constexpr float kLift = 12.f, kLimit = 60000.f;
  typedef half_t v8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mad(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};
template <>
struct Matrix<bfloat_t> {
  static constexpr uint32_t kNoNumber = 0x7f80u;
  static constexpr float kLift = 0.f, kLimit = 1e6f;      // the range of a float
  typedef bfloat_t v8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mad(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef T two __attribute__((ext_vector_type(2)));
  two v;
  v[0] = (T)a;
  v[1] = (T)b;
  return __builtin_bit_cast(uint32_t, v);
}

// Both halves of a word, those that are no finite numbers as 0.
template <typename T>
__device__ __forceinline__ uint32_t numbers(uint32_t w) {
  constexpr uint32_t e = Matrix<T>::kNoNumber;
  return ((w & e) == e ? 0u : w & 0xffffu) | ((w & (e << 16)) == (e << 16) ? 0u : w & 0xffff0000u);
}

// D elements of a token are 16 lanes of D / 16 elements: N words of each
template <int N>
struct Words {
  uint32_t w[N];
};
template <int N>
using WordsAtOnce = uint32_t __attribute__((ext_vector_type(N % 4 == 0 ? 4 : N % 2 == 0 ? 2 : 1)));
template <int N>
__device__ __forceinline__ Words<N> load_words(const char* p) {
  typedef WordsAtOnce<N> some;
  constexpr int A = sizeof(some) / 4;
  Words<N> r;
#pragma unroll
  for (int i = 0; i < N / A; ++i) {
    const some s = reinterpret_cast<const some*>(p)[i];
#pragma unroll
    for (int j = 0; j < A; ++j) r.w[i * A + j] = s[j];
  }
  return r;
}
template <int N>
__device__ __forceinline__ void store_words(char* p, const uint32_t (&w)[N]) {
  typedef WordsAtOnce<N> some;
  constexpr int A = sizeof(some) / 4;
#pragma unroll
  for (int i = 0; i < N / A; ++i) {
    some s;
#pragma unroll
    for (int j = 0; j < A; ++j) s[j] = w[i * A + j];
    reinterpret_cast<some*>(p)[i] = s;
  }
}

// The weights of a row relative to the score m add up to s, which is 0 only where the row has no score: the largest counts 1 or more.  A row whose scores are
// NaN has a NaN for a sum and maybe no m, so it is the sum that tells, and the NaN that ends up in the result.
__device__ __forceinline__ float one_over(float s) { return s == 0.f ? 0.f : 1.f / s; }
// The logarithm of the sum of exp(scale x) over the row.
template <typename T>
__device__ __forceinline__ float log_sum(float m, float s, float scale) {
  return s == 0.f ? -INFINITY : m * scale + (__builtin_amdgcn_logf(s) - Matrix<T>::kLift) * 0.69314718055994530942f;
}

// The largest value of the four lanes of a row (16 lanes apart).
__device__ __forceinline__ float row_max(float x) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const uint32_t w = __float_as_uint(x);
  const u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(w, w, false, false));
  const uint32_t v = __float_as_uint(fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1])));
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(v, v, false, false));
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// What a wavefront has of its rows: the weighted values, the weights' sum, and the score `top` they are relative to: a weight is
// 2^((x - top) scale + lift), formed as 2^(x scale + from).  from is rounded to a step of its size, which all weights of the row share: nothing next to the
// rounding of the scores themselves, but beside products of more than kHuge it would come to more than the weights' range (and the products may be past the floats).  There
// top is taken from the scores first and from is the lift.
constexpr float kHuge = 65536.f;      // steps of 2^-7: weights within 0.3 % of what they should be
template <int MT, int DV>
struct Rows {
  f32x4 o[MT][DV];
  float sum[MT], top[MT], from[MT];      // sum: of the lane's own tokens
  bool huge, waiting;      // waiting: some row has no score yet
  __device__ __forceinline__ void clear() {
    huge = false;
    waiting = true;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      top[mt] = -INFINITY;
      from[mt] = 0.f;
      sum[mt] = 0.f;
#pragma unroll
      for (int j = 0; j < DV; ++j) o[mt][j] = f32x4{0, 0, 0, 0};
    }
  }
};

// The scores of one step of 32 tokens for 16 * MT rows, in the lanes that the value product wants their weights in: with 16 x 16 x 32 matrix instructions lane l
// holds row l % 16 of Q and, of a result of K Q^T, the tokens 4 (l / 16) ... + 3; if the first 16 tokens of a step are numbered 8 (m / 4) + m % 4 and the second 16
// four more, lane group l / 16 holds the weights of the tokens 8 (l / 16) ... + 7, which is the operand of V^T P^T.
template <int MT>
using Scores = f32x4[MT][2];

template <typename T, int D, int MT>
__device__ __forceinline__ void score(const u32x4 (&q)[MT][D / 32], const u32x4 (&k)[2][D / 32], Scores<MT>& s) {
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    s[mt][0] = s[mt][1] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
      s[mt][0] = Matrix<T>::mad(k[0][kk], q[mt][kk], s[mt][0]);
      s[mt][1] = Matrix<T>::mad(k[1][kk], q[mt][kk], s[mt][1]);
    }
  }
}

// Tokens that a row does not see have no score.
template <int MT>
__device__ __forceinline__ void mask(Scores<MT>& s, const uint32_t (&seen)[MT]) {
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int i = 0; i < 8; ++i) s[mt][i / 4][i % 4] = (seen[mt] >> i) & 1 ? s[mt][i / 4][i % 4] : -INFINITY;
}

// The weights of a step, rounded for the value product, and their sum.  They are formed with the `top` there is: only where a lane's weights come to more than kLimit,
// or a row has none, does top follow the largest score, with an exchange between lanes and a scaling of o, and the weights are formed again.  That is the first step with
// a score and few after it (but all steps of a wavefront with a row that sees nothing, of which only nodes make some); all others look for no maximum at all.
template <typename T, int MT, int DV>
__device__ __forceinline__ void weigh(Rows<MT, DV>& r, Scores<MT>& s, float scale_log2, u32x4 (&w)[MT]) {
  constexpr float kLift = Matrix<T>::kLift;
  float x[MT][8], add[MT];
  auto form = [&]() {
    if (r.huge) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[mt][i] = (s[mt][i / 4][i % 4] - (r.top[mt] == -INFINITY ? 0.f : r.top[mt])) * scale_log2 + r.from[mt];
    } else {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[mt][i] = __builtin_fmaf(s[mt][i / 4][i % 4], scale_log2, r.from[mt]);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[mt][i] = __builtin_amdgcn_exp2f(x[mt][i]);
      add[mt] = ((x[mt][0] + x[mt][1]) + (x[mt][2] + x[mt][3])) + ((x[mt][4] + x[mt][5]) + (x[mt][6] + x[mt][7]));
    }
  };
  form();
  bool behind = false;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) behind = behind || add[mt] > Matrix<T>::kLimit;
  if (r.waiting || __any(behind)) {
    bool huge = false, waiting = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float most = s[mt][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) most = fmaxf(most, s[mt][i / 4][i % 4]);
      const float next = fmaxf(r.top[mt], row_max(most));
      const float less = r.top[mt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((r.top[mt] - next) * scale_log2);
      r.top[mt] = next;
      huge = huge || (next != -INFINITY && __builtin_fabsf(next) * scale_log2 > kHuge);
      r.sum[mt] *= less;
#pragma unroll
      for (int j = 0; j < DV; ++j) r.o[mt][j] *= less;
    }
    r.huge = __any(huge);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
      r.from[mt] = r.top[mt] == -INFINITY ? 0.f : r.huge ? kLift : __builtin_fmaf(-r.top[mt], scale_log2, kLift);
    form();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) waiting = waiting || (r.top[mt] == -INFINITY && add[mt] == add[mt]);      // (a row of NaN waits for nothing)
    r.waiting = __any(waiting);
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    r.sum[mt] += add[mt];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[mt][i] = pack2<T>(x[mt][2 * i], x[mt][2 * i + 1]);
  }
}

// How the tokens are dealt out.  For every kv head and tile of rows a launch has `slots` workgroups; all take parts of the same number of steps, the smallest
// with which the parts of all sequences fit (a sequence has at least one, which writes the zeros of a row that sees nothing).  With parts of c steps the
// sequences need at least total / c and less than total / c + batch, so c is between total / slots and total / (slots - batch + 1); a batch of up
// to 64 looks for it there, 64 values at a time, a larger one takes the latter.  The lengths are on the device, so every workgroup works this out for itself.
struct Share {
  int b, len, first, last;      // sequence (-1: nothing is left for this slot), its tokens in the cache, steps
  int part, parts;              // of the sequence
};

__device__ __forceinline__ int tokens_of(const AttentionArgs& a, int b) { return min(max(a.lens[b], 0), a.cache.pages_per_seq * a.cache.page); }
__device__ __forceinline__ int steps_of(int tokens) { return (int)(((uint32_t)tokens + kAttTile - 1) / kAttTile); }

__device__ __forceinline__ Share share_in(const AttentionArgs& a, int slot) {
  const int lane = threadIdx.x & 63, extra = steps_of(a.seen_nodes);
  if (a.batch == 1) {
    const int len = tokens_of(a, 0), steps = steps_of(len) + extra;
    const int each = max((steps + a.slots - 1) / a.slots, a.least), parts = max(1, (steps + each - 1) / each);
    return {slot < parts ? 0 : -1, len, slot * each, min((slot + 1) * each, steps), slot, parts};
  }
  int64_t total = 0;
  int len = 0;
  for (int first = 0; first < a.batch; first += 64) {
    const int b = first + lane;
    len = b < a.batch ? tokens_of(a, b) : 0;
    total += b < a.batch ? steps_of(len) + extra : 0;
  }
#pragma unroll
  for (int i = 1; i < 64; i *= 2) total += __shfl_xor(total, i);
  const int64_t over = a.slots - a.batch + 1;
  int each = max((int)((total + over - 1) / over), a.least);      // steps of a part; it fits
  if (a.batch <= 64 && a.slots > a.batch) {
    const int steps = lane < a.batch ? steps_of(len) + extra : 0, from = max((int)((total + a.slots - 1) / a.slots), a.least);
    const int mine = from + (int)((int64_t)(each - from) * lane / 64);
    const float by = 1.0f / (float)mine;      // steps are below 2^26 and the quotient is raised by a step: at most one part too many is counted
    int parts = 0;
    for (int b = 0; b < a.batch; ++b) {
      const int s = __builtin_amdgcn_readlane(steps, b);
      parts += max(1, (int)((float)(s - 1) * by + 1.0f + 1.0f / 256));
    }
    const uint64_t fits = __ballot(parts <= a.slots);
    if (fits != 0) each = __builtin_amdgcn_readlane(mine, __ffsll((unsigned long long)fits) - 1);
  }
  int before = 0;
  for (int first = 0; first < a.batch; first += 64) {
    const int b = first + lane;
    if (a.batch > 64) len = b < a.batch ? tokens_of(a, b) : 0;
    const int steps = steps_of(len) + extra, n = b < a.batch ? max(1, (steps + each - 1) / each) : 0;
    int upto = n;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
      const int v = __shfl_up(upto, i);
      if (lane >= i) upto += v;
    }
    upto += before;
    const uint64_t mine = __ballot(slot < upto && slot >= upto - n);
    if (mine != 0) {
      const int l = __ffsll((unsigned long long)mine) - 1, part = slot - __shfl(upto - n, l), s = __shfl(steps, l);
      return {first + l, __shfl(len, l), part * each, min((part + 1) * each, s), part, __shfl(n, l)};
    }
    before = __shfl(upto, 63);
  }
  return {-1, 0, 0, 0, 0, 0};
}

// The same in scalar registers: every lane has found the same.
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Share share_of(const AttentionArgs& a, int slot) {
  const Share s = share_in(a, slot);
  return {scalar(s.b), scalar(s.len), scalar(s.first), scalar(s.last), scalar(s.part), scalar(s.parts)};
}

// Where the rows of a workgroup's part lie among the parts.
__device__ __forceinline__ int64_t part_row(const AttentionArgs& a, int slot, int h, int row_tile, int rows_of_tile) {
  return (((int64_t)slot * a.kv_heads + h) * a.row_tiles + row_tile) * rows_of_tile;
}

// The nodes among t ... t + 7 that a node sees, a bit each.
__device__ __forceinline__ uint32_t seen_of(const AttentionArgs& a, int b, int node, int t) {
  if (node < 0 || t >= a.seen_nodes) return 0u;
  if (a.mask == nullptr) return node < t ? 0u : node - t >= 7 ? 0xffu : (2u << (node - t)) - 1u;
  return (uint32_t)(a.mask[b * a.mask_stride + node * a.words + (t >> 6)] >> (t & 63)) & 0xffu;
}

// The queries of a wavefront's 16 * MT rows from row `first` on, and their nodes (-1: no row).
template <int D, int MT>
__device__ __forceinline__ void load_queries(const AttentionArgs& a, int b, int h, int first, u32x4 (&q)[MT][D / 32], int (&node)[MT]) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = first + mt * 16 + n;
    node[mt] = -1;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) q[mt][kk] = u32x4{0, 0, 0, 0};
    if (r < a.rows) {
      node[mt] = a.by_group.of(r);
      const char* p = a.q.data + 2 * (b * a.q.batch_stride + node[mt] * a.q.token_stride + (h * a.group + r - node[mt] * a.group) * a.q.head_stride + 8 * g);
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) q[mt][kk] = (*reinterpret_cast<const u32x4*>(p + 64 * kk) & a.keep) ^ a.sign;
    }
  }
}

// Where token lane % 32 of a step lies.  The page id is asked for a step or more before the place is needed.  Places are offsets in bytes from the start of the
// head, in page 0 of the cache (a step of the context) or in node 0, separately for keys and values; a token that is not there has the place of one that is.
// The steps past the last that a loop asks for ahead, so that its loads are the same in number every time, are all at the start of page 0.
struct Lookup {
  int page;
  uint32_t token;
};
// (a choice between values: between variables, which it is in a lambda, it would be one of addresses, and put them into memory)
__device__ __forceinline__ const char* either(bool first, const char* a, const char* b) { return first ? a : b; }
struct Place {
  int64_t k, v;
  bool there;
};
__device__ __forceinline__ Lookup ask(const AttentionArgs& a, const Share& s, int old_steps, int step) {
  Lookup l{s.b, (uint32_t)step * kAttTile + (threadIdx.x & (kAttTile - 1))};
  if (step >= s.last) return l;
  if (step >= old_steps) {
    l.token -= (uint32_t)old_steps * kAttTile;
  } else if (a.cache.table != nullptr) {
    l.page = a.cache.table[s.b * a.cache.table_stride + a.cache.by_page.of(min(l.token, (uint32_t)s.len - 1))];      // (a step of the context has a token)
  }
  return l;
}
__device__ __forceinline__ Place place_of(const AttentionArgs& a, const Share& s, int old_steps, int step, const Lookup& l) {
  Place p{0, 0, false};
  if (step >= s.last) return p;
  if (step >= old_steps) {
    p.there = l.token < (uint32_t)a.seen_nodes;
    const int64_t t = p.there ? l.token : 0;
    p.k = 2 * t * a.k_new.token_stride;
    p.v = 2 * t * a.v_new.token_stride;
  } else {
    p.there = l.token < (uint32_t)s.len && (uint32_t)l.page < (uint32_t)a.cache.pages;
    const int64_t at = l.page * a.cache.page_stride + (int64_t)(l.token - a.cache.by_page.of(l.token) * (uint32_t)a.cache.page) * a.cache.token_stride;
    p.k = p.v = p.there ? 2 * at : 0;
  }
  return p;
}

// A node may be seen by some rows only, and for the others its values may be anything.  In the value product they would meet weights of zero, so what is no finite number
// leaves that product, and when all is added up the rows that see it add it as it is: a weight above zero changes no infinity and no NaN.
// Of the steps, those that this wavefront took in its turn.  PLAIN: a lane's values are 4 DV g + j in o[j % DV][j / DV]; else 16 (j / 4) + 4 g + j % 4 in o[j / 4][j % 4].
template <typename T, int D, int MT, bool PLAIN>
__device__ __forceinline__ void add_odd_values(const AttentionArgs& a, Rows<MT, D / 16>& r, const Share& s, int old_steps, const char* new_v, const int (&node)[MT], int turn,
                                               int turns) {
  constexpr int DV = D / 16;
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll 1
  for (int t = max(s.first - old_steps, 0) * kAttTile; t < min((s.last - old_steps) * kAttTile, a.seen_nodes); ++t) {
    if ((old_steps + t / kAttTile - s.first) % turns != turn) continue;
    const T* values = reinterpret_cast<const T*>(new_v) + t * a.v_new.token_stride;
    bool sees[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) sees[mt] = (seen_of(a, s.b, node[mt], t & ~7) >> (t & 7)) & 1;
#pragma unroll
    for (int j = 0; j < 4 * DV; ++j) {
      const float value = (float)values[PLAIN ? 4 * DV * g + j : 16 * (j / 4) + 4 * g + j % 4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        if (sees[mt] && !__builtin_isfinite(value)) r.o[mt][PLAIN ? j % DV : j / 4][PLAIN ? j / DV : j % 4] += value;
    }
  }
}

// The kernel for few rows.  One workgroup: up to 16 * MT rows (node, query head of one kv head) of one sequence over one part of its tokens; its wavefronts
// take steps of 32 tokens in turns and meet at the end.  K and V go from memory to the registers they are used from: K as it lies is an operand,
// V is loaded as it lies, D / 16 elements of 8 tokens to a lane, and turned inside the lane, 16 bits at a time.
// The weights are rounded to the type of V for the value product (their sum is not): half a step of each, so the error is a mean of independent
// roundings, below the one rounding of the result.
template <typename T, int D, int MT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, D <= 128 ? 2 : 1) tree_attention_kernel(const AttentionArgs a) {
  constexpr int KK = D / 32, DV = D / 16, N = DV / 2, R = 16 * MT;
  constexpr int PER = 4 * DV / WAVES;      // of a lane's 4 DV results, which lie side by side, what a wavefront adds up in the end
  __shared__ float sums[WAVES][4 * DV * MT][64];
  __shared__ float2 tops[WAVES][MT][16];
  __shared__ __align__(16) int64_t places[WAVES][2][2][kAttTile];      // [..][turn][keys, values][token]
  const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  uint32_t id = blockIdx.x;
  const int h = id % a.kv_heads;
  id /= a.kv_heads;
  const int row_tile = id % a.row_tiles, slot = id / a.row_tiles;
  const Share share = share_of(a, slot);
  if (share.b < 0) return;
  const int b = share.b, old_steps = steps_of(share.len), last = share.last;
  if (share.part == 0 && h == 0 && row_tile == 0 && threadIdx.x == 0 && a.places != nullptr) a.places[b] = make_int2(slot, share.parts);

  u32x4 q[MT][KK];
  int node[MT];
  int step = share.first + wave;
  Lookup next = ask(a, share, old_steps, step);
  load_queries<D, MT>(a, b, h, row_tile * R, q, node);
  Rows<MT, DV> rows;
  rows.clear();
  const int k_token = 8 * (n >> 2) + (n & 3);      // of the first 16; the second are 4 further
  const char *cache_k = a.cache.k + 2 * h * a.cache.head_stride, *cache_v = a.cache.v + 2 * h * a.cache.head_stride;
  const char *new_k = a.k_new.data + 2 * (b * a.k_new.batch_stride + h * a.k_new.head_stride),
             *new_v = a.v_new.data + 2 * (b * a.v_new.batch_stride + h * a.v_new.head_stride);
  struct Tokens {
    u32x4 k[2][KK];
    Words<N> v[8];
    uint32_t there;
  };
  // Asks for the tokens of a step, and for the places of the one behind it.  The places pass through LDS, from the lane that looked one up to those that load
  // from it; a wavefront's own accesses there are in order.
  auto load = [&](int step, int turn, Tokens& x) {
    const bool old = step < old_steps || step >= last;
    const Place mine = place_of(a, share, old_steps, step, next);
    int64_t(*table)[kAttTile] = places[wave][turn];
    if (lane < kAttTile) {
      table[0][lane] = mine.k;
      table[1][lane] = mine.v;
    }
    x.there = (uint32_t)__ballot(mine.there);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const char *base_k = either(old, cache_k, new_k) + 16 * g, *base_v = either(old, cache_v, new_v) + 2 * DV * n;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const char* p = base_k + table[0][k_token + 4 * half];
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) x.k[half][kk] = *reinterpret_cast<const u32x4*>(p + 64 * kk);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i] = load_words<N>(base_v + table[1][8 * g + i]);
    next = ask(a, share, old_steps, step + WAVES);
  };
  bool odd = false;      // among the values of nodes is something that is no finite number
  auto attend = [&](int step, Tokens& x) {
    const bool old = step < old_steps, all = old && x.there == 0xffffffffu;
    uint32_t seen[MT] = {};
    const int t0 = (step - old_steps) * kAttTile;
    Scores<MT> s;
    u32x4 w[MT];
    score<T, D, MT>(q, x.k, s);
    if (!all) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        seen[mt] = (x.there >> (8 * g)) & 0xffu;
        if (!old) seen[mt] &= seen_of(a, b, node[mt], t0 + 8 * g);
      }
      mask<MT>(s, seen);
    }
    weigh<T, MT, DV>(rows, s, a.scale_log2, w);
    if (!all) {
      // a token that is not there was read from a place that is, and counts as zeros
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const uint32_t is = (x.there >> (8 * g + i)) & 1 ? x.v[i].w[j] : 0u, number = old ? is : numbers<T>(is);
          odd = odd || number != is;
          x.v[i].w[j] = number;
        }
    }
#pragma unroll
    for (int j = 0; j < DV; ++j) {
      u32x4 t;
#pragma unroll
      for (int i = 0; i < 4; ++i) t[i] = __builtin_amdgcn_perm(x.v[2 * i + 1].w[j / 2], x.v[2 * i].w[j / 2], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) rows.o[mt][j] = Matrix<T>::mad(t, w[mt], rows.o[mt][j]);
    }
  };
  Tokens x;
  for (int turn = 0; step < last; step += WAVES, turn ^= 1) {
    load(step, turn, x);
    attend(step, x);
  }

  if (__any(odd)) add_odd_values<T, D, MT, true>(a, rows, share, old_steps, new_v, node, wave, WAVES);
  // the wavefronts' rows meet: each wavefront adds up its part of the elements
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float s = rows.sum[mt];
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (g == 0) tops[wave][mt][n] = make_float2(rows.top[mt], s);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < DV; ++j) sums[wave][(mt * 4 + i) * DV + j][lane] = rows.o[mt][j][i];
  }
  __syncthreads();
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = row_tile * R + mt * 16 + n;
    float m = -INFINITY, s = 0.f, f[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, tops[w][mt][n].x);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      f[w] = tops[w][mt][n].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((tops[w][mt][n].x - m) * a.scale_log2);
      s += tops[w][mt][n].y * f[w];
    }
    float e[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      e[j] = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) e[j] += sums[w][mt * 4 * DV + wave * PER + j][lane] * f[w];
    }
    if (r >= a.rows) continue;
    const int d = 4 * DV * g + wave * PER;
    if (share.parts == 1) {
      const float by = one_over(s);
      uint32_t words[PER / 2];
#pragma unroll
      for (int j = 0; j < PER / 2; ++j) words[j] = pack2<T>(e[2 * j] * by, e[2 * j + 1] * by);
      const int head = h * a.group + r - node[mt] * a.group;
      store_words(a.out.data + 2 * (b * a.out.batch_stride + node[mt] * a.out.token_stride + head * a.out.head_stride + d), words);
      if (a.lse != nullptr && g == 0 && wave == 0) a.lse[((int64_t)b * a.nodes + node[mt]) * (a.kv_heads * a.group) + head] = log_sum<T>(m, s, a.scale);
    } else {
      const int64_t row = part_row(a, slot, h, row_tile, R) + mt * 16 + n;
      uint32_t words[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) words[j] = __builtin_bit_cast(uint32_t, e[j]);
      if (m != -INFINITY) store_words(reinterpret_cast<char*>(a.part + row * D + d), words);
      if (g == 0 && wave == 0) a.stats[row] = make_float2(m, s);
    }
  }
}

// The parts of a row meet: one wavefront to a row.  Tops first, then sums of eight parts at a time, so that their loads are on the way together.  (A part without a
// top is not read.  It may have a NaN for a sum: then so has the row, and all of the result is NaN.)
template <typename T, int D>
__global__ void __launch_bounds__(256) tree_attention_join_kernel(const AttentionArgs a, int rows_of_tile, Divide by_rows, Divide by_heads, Divide by_tile, uint32_t all_rows) {
  const int lane = threadIdx.x & 63;
  const uint32_t id = blockIdx.x * 4 + (threadIdx.x >> 6);      // [batch][kv head][row]
  if (id >= all_rows) return;
  const uint32_t bh = by_rows.of(id), r = id - bh * a.rows, b = by_heads.of(bh), h = bh - b * a.kv_heads, row_tile = by_tile.of(r);
  const int2 place = a.places[b];
  const int parts = place.y;
  if (parts == 1) return;      // its workgroup has written the result
  const int64_t first = part_row(a, place.x, h, row_tile, rows_of_tile) + (r - row_tile * rows_of_tile), step = (int64_t)a.kv_heads * a.row_tiles * rows_of_tile;
  constexpr int P = D >= 128 ? D / 128 : 1;      // a lane has two neighbouring elements of every 128 (D below 128: the first D / 2 lanes)
  const int at = D >= 128 || lane < D / 2 ? lane * 2 : 0;
  float m = -INFINITY, s = 0.f, e[P * 2] = {};
  for (int p0 = 0; p0 < parts; p0 += 64) {
    const float2 mine = p0 + lane < parts ? a.stats[first + (p0 + lane) * step] : make_float2(-INFINITY, 0.f);
    float top = mine.x;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
    const float next = fmaxf(m, top), less = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - next) * a.scale_log2);
    const float f = mine.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mine.x - next) * a.scale_log2);
    float add = f * mine.y;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) add += __shfl_xor(add, i);
    m = next;
    s = s * less + add;
#pragma unroll
    for (int j = 0; j < 2 * P; ++j) e[j] *= less;
    const int here = min(64, parts - p0);
    for (int i0 = 0; i0 < here; i0 += 8) {
      float2 v[8][P];
      float by[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int part = min(i0 + i, here - 1);
        by[i] = i0 + i < here ? __shfl(f, part) : 0.f;
        const float* p = a.part + (first + (p0 + part) * step) * D + at;
#pragma unroll
        for (int j = 0; j < P; ++j) v[i][j] = *reinterpret_cast<const float2*>(p + j * 128);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < P; ++j) {      // (a part that its rows saw nothing of has not been written)
          e[2 * j] += by[i] == 0.f ? 0.f : by[i] * v[i][j].x;
          e[2 * j + 1] += by[i] == 0.f ? 0.f : by[i] * v[i][j].y;
        }
    }
  }
  const float by = one_over(s);
  const int node = a.by_group.of(r), head = h * a.group + r - node * a.group;
  char* out = a.out.data + 2 * (b * a.out.batch_stride + node * a.out.token_stride + head * a.out.head_stride + at);
  if (D >= 128 || lane < D / 2)
#pragma unroll
    for (int j = 0; j < P; ++j) *reinterpret_cast<uint32_t*>(out + 256 * j) = pack2<T>(e[2 * j] * by, e[2 * j + 1] * by);
  if (a.lse != nullptr && lane == 0) a.lse[((int64_t)b * a.nodes + node) * (a.kv_heads * a.group) + head] = log_sum<T>(m, s, a.scale);
}

// The kernel for many rows: WAVES wavefronts with 16 * MT rows each take every step together.  K and V of a step are loaded once for all of them and kept
// in LDS, two steps in turns: the next step's are asked for before this one's products and written behind them.
//   K: pieces of 8 elements [D / 8][32 tokens], the tokens' places exclusive-or the piece's number, so that neither the writing (a row of the
//      cache at a time) nor the reading (16 tokens of four pieces) meets itself in a bank;
//   V: turned while it is written: [4 groups of 8 tokens][D] of 16 bytes, as the value product reads it.
// A lane's results are the values 16 j + 4 g ... + 3 of its row, j < D / 16.
template <typename T, int D, int MT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, D <= 128 && MT <= 2 ? 2 : 1) tree_attention_wide_kernel(const AttentionArgs a) {
  constexpr int KK = D / 32, DV = D / 16, R = 16 * MT * WAVES, THREADS = WAVES * 64;
  constexpr int U = (4 * D + THREADS - 1) / THREADS;      // units of 16 bytes of K, and of V, to a thread
  __shared__ __align__(16) char lds_k[2][4 * D * 16], lds_v[2][4 * D * 16];
  __shared__ __align__(16) int64_t places[2 * WAVES][2][kAttTile];      // [step][keys, values][token]
  __shared__ uint32_t lds_there[2 * WAVES], lds_odd;
  const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  uint32_t id = blockIdx.x;
  const int h = id % a.kv_heads;
  id /= a.kv_heads;
  const int row_tile = id % a.row_tiles, slot = id / a.row_tiles;
  const Share share = share_of(a, slot);
  if (share.b < 0) return;
  const int b = share.b, old_steps = steps_of(share.len), first = share.first, last = share.last;
  if (share.part == 0 && h == 0 && row_tile == 0 && threadIdx.x == 0 && a.places != nullptr) a.places[b] = make_int2(slot, share.parts);

  // Places are looked up for as many steps at a time as there are wavefronts, one by each, at least that many steps before they are needed: one wavefront that
  // does it every step keeps the others waiting at the barrier.
  auto keep_places = [&](int step, const Lookup& l) {
    const Place mine = place_of(a, share, old_steps, step, l);
    if (lane < kAttTile) {
      places[(step - first) & (2 * WAVES - 1)][0][lane] = mine.k;
      places[(step - first) & (2 * WAVES - 1)][1][lane] = mine.v;
    }
    const uint32_t there = (uint32_t)__ballot(mine.there);
    if (lane == 0) lds_there[(step - first) & (2 * WAVES - 1)] = there;
  };
  keep_places(first + wave, ask(a, share, old_steps, first + wave));
  if (threadIdx.x == 0) lds_odd = 0;
  u32x4 q[MT][KK];
  int node[MT];
  load_queries<D, MT>(a, b, h, row_tile * R + wave * 16 * MT, q, node);
  const bool works = row_tile * R + wave * 16 * MT < a.rows;      // a wavefront without rows only loads
  Rows<MT, DV> rows;
  rows.clear();

  // What this thread loads of a step: unit u of K is piece u % (D / 8) of token u / (D / 8); of V it is the elements 2 (u % (D / 2)) and the next of four tokens.
  const char *cache_k = a.cache.k + 2 * h * a.cache.head_stride, *cache_v = a.cache.v + 2 * h * a.cache.head_stride;
  const char *new_k = a.k_new.data + 2 * (b * a.k_new.batch_stride + h * a.k_new.head_stride),
             *new_v = a.v_new.data + 2 * (b * a.v_new.batch_stride + h * a.v_new.head_stride);
  struct Units {
    u32x4 k[U];
    uint32_t v[U][4];
  };
  auto load = [&](int step, Units& x) {
    const bool old = step < old_steps || step >= last;
    const char *base_k = either(old, cache_k, new_k), *base_v = either(old, cache_v, new_v);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = min((int)threadIdx.x + i * THREADS, 4 * D - 1);
      x.k[i] = *reinterpret_cast<const u32x4*>(base_k + places[(step - first) & (2 * WAVES - 1)][0][u / (D / 8)] + 16 * (u % (D / 8)));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x.v[i][j] = *reinterpret_cast<const uint32_t*>(base_v + places[(step - first) & (2 * WAVES - 1)][1][4 * (u / (D / 2)) + j] + 4 * (u % (D / 2)));
    }
  };
  auto there_in = [&](int step) { return (uint32_t)scalar((int)lds_there[(step - first) & (2 * WAVES - 1)]); };
  auto keep = [&](int step, Units& x) {
    const uint32_t there = there_in(step);
    const bool old = step < old_steps;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = threadIdx.x + i * THREADS;
      if (4 * D % THREADS != 0 && u >= 4 * D) continue;
      const int four = u / (D / 2), d = 2 * (u % (D / 2));
      if (!old || there != 0xffffffffu) {      // (as in the kernel for few rows)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t is = (there >> (4 * four + j)) & 1 ? x.v[i][j] : 0u, number = old ? is : numbers<T>(is);
          odd = odd || number != is;
          x.v[i][j] = number;
        }
      }
      const int token = u / (D / 8), place = ((token >> 2) & 1) * 16 + 4 * (token >> 3) + (token & 3), piece = u % (D / 8);      // as score() numbers the tokens
      *reinterpret_cast<u32x4*>(lds_k[step & 1] + (piece * kAttTile + (place ^ (piece & 15))) * 16) = x.k[i];
      char* to = lds_v[step & 1] + ((four >> 1) * D + d) * 16 + (four & 1) * 8;
      const uint32_t* v = x.v[i];
      *reinterpret_cast<uint2*>(to) = make_uint2(__builtin_amdgcn_perm(v[1], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[2], 0x05040100u));
      *reinterpret_cast<uint2*>(to + 16) = make_uint2(__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u));
    }
    if (odd) lds_odd = 1;
  };
  auto attend = [&](int step) {
    u32x4 w[MT], values[DV], k[2][KK];
    Scores<MT> s;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        k[half][kk] = *reinterpret_cast<const u32x4*>(lds_k[step & 1] + ((4 * kk + g) * kAttTile + half * 16 + (n ^ ((4 * kk + g) & 15))) * 16);
    score<T, D, MT>(q, k, s);
    // V is read before the weights are formed, so that it is there when they are (192 -> 179 us)
#pragma unroll
    for (int j = 0; j < DV; ++j) values[j] = *reinterpret_cast<const u32x4*>(lds_v[step & 1] + (g * D + 16 * j + n) * 16);
    const uint32_t there = there_in(step);
    if (step >= old_steps || there != 0xffffffffu) {
      uint32_t seen[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        seen[mt] = (there >> (8 * g)) & 0xffu;
        if (step >= old_steps) seen[mt] &= seen_of(a, b, node[mt], (step - old_steps) * kAttTile + 8 * g);
      }
      mask<MT>(s, seen);
    }
    weigh<T, MT, DV>(rows, s, a.scale_log2, w);
#pragma unroll
    for (int j = 0; j < DV; ++j)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) rows.o[mt][j] = Matrix<T>::mad(values[j], w[mt], rows.o[mt][j]);
  };

  __syncthreads();
  Units x;
  if (first < last) {
    load(first, x);
    keep(first, x);
  }
  __syncthreads();
  for (int step = first; step < last; ++step) {
    const bool ahead = ((step - first) & (WAVES - 1)) == 0;
    Lookup after{};
    if (ahead) after = ask(a, share, old_steps, step + WAVES + wave);
    load(step + 1, x);
    if (works) attend(step);
    keep(step + 1, x);
    if (ahead) keep_places(step + WAVES + wave, after);
    __syncthreads();
  }
  if (!works) return;
  if (lds_odd) add_odd_values<T, D, MT, false>(a, rows, share, old_steps, new_v, node, 0, 1);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int in_tile = wave * 16 * MT + mt * 16 + n, r = row_tile * R + in_tile;
    float s = rows.sum[mt];
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (r >= a.rows) continue;
    const float m = rows.top[mt];
    if (share.parts == 1) {
      const float by = one_over(s);
      const int head = h * a.group + r - node[mt] * a.group;
      char* out = a.out.data + 2 * (b * a.out.batch_stride + node[mt] * a.out.token_stride + head * a.out.head_stride + 4 * g);
#pragma unroll
      for (int j = 0; j < DV; ++j)
        *reinterpret_cast<uint2*>(out + 32 * j) = make_uint2(pack2<T>(rows.o[mt][j][0] * by, rows.o[mt][j][1] * by), pack2<T>(rows.o[mt][j][2] * by, rows.o[mt][j][3] * by));
      if (a.lse != nullptr && g == 0) a.lse[((int64_t)b * a.nodes + node[mt]) * (a.kv_heads * a.group) + head] = log_sum<T>(m, s, a.scale);
    } else {
      const int64_t row = part_row(a, slot, h, row_tile, R) + in_tile;
      if (m != -INFINITY)
#pragma unroll
        for (int j = 0; j < DV; ++j) *reinterpret_cast<f32x4*>(a.part + row * D + 16 * j + 4 * g) = rows.o[mt][j];
      if (g == 0) a.stats[row] = make_float2(m, s);
    }
  }
}

}  // namespace dpllm
