// Attention of a few drafted tokens (the nodes of a tree) over a paged cache and over one another.
//
// For the row (node i, query head h) of a sequence: x_t = scale q . k_t over the tokens t of the cache and those nodes that the
// mask of i names, out = sum_t exp(x_t - m) v_t / sum_t exp(x_t - m), m the largest x_t; a row that sees nothing is zero.
#pragma once
#include "token_common.hpp"

namespace dpllm {

constexpr int kAttWaves = 4;        // wavefronts of a workgroup of the kernel for few rows
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
  // weights reach the matrix pipe as 2^12 times what they are: with the slack of a row's top at most 2^15, and rounded to multiples of
  // 2^-24, as a half below 2^-14 is, only where they are below 2^-26 of the top's
  static constexpr float kLift = 12.f, kSlack = 3.f;
  typedef half_t v8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mad(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};
template <>
struct Matrix<bfloat_t> {
  static constexpr uint32_t kNoNumber = 0x7f80u;
  static constexpr float kLift = 0.f, kSlack = 8.f;      // the range of a float
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

// The logarithm of the sum of exp(scale x) over a row whose weights relative to the score m add up to s.
template <typename T>
__device__ __forceinline__ float log_sum(float m, float s, float scale) {
  return m == -INFINITY ? m : m * scale + (__builtin_amdgcn_logf(s) - Matrix<T>::kLift) * 0.69314718055994530942f;
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
// 2^((x - top) scale + lift), formed as 2^(x scale + from).
template <int MT, int DV>
struct Rows {
  f32x4 o[MT][DV];
  float sum[MT], top[MT], from[MT];      // sum: of the lane's own tokens
  float limit[MT];                       // the score from which on top has to follow
  bool huge;                             // some top times scale / ln 2 may be past the floats though the scores are not
  __device__ __forceinline__ void clear(float lift) {
    huge = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      top[mt] = limit[mt] = -INFINITY;
      from[mt] = lift;
      sum[mt] = 0.f;
#pragma unroll
      for (int j = 0; j < DV; ++j) o[mt][j] = f32x4{0, 0, 0, 0};
    }
  }
};

// The weights of one step of 32 tokens for 16 * MT rows, in the lanes that the value product wants them in: with 16 x 16 x 32 matrix instructions lane l
// holds row l % 16 of Q and, of a result of K Q^T, the tokens 4 (l / 16) ... + 3; if the first 16 tokens of a step are numbered 8 (m / 4) + m % 4 and the second 16
// four more, lane group l / 16 holds the weights of the tokens 8 (l / 16) ... + 7, which is the operand of V^T P^T.
// `top` follows the largest score only when that has left it behind by 2^kSlack: in most steps no row's has, and the exchange between
// lanes and the scaling of o are skipped.  ALL: every row sees every token.
template <typename T, int D, int MT, bool ALL>
__device__ __forceinline__ void weigh(Rows<MT, D / 16>& r, const u32x4 (&q)[MT][D / 32], const u32x4 (&k)[2][D / 32], float scale_log2,
                                      const uint32_t (&seen)[MT], u32x4 (&w)[MT]) {
  constexpr int KK = D / 32, DV = D / 16;
  constexpr float kLift = Matrix<T>::kLift, kSlack = Matrix<T>::kSlack;
  f32x4 s[MT][2];
  float most[MT];
  bool behind = false;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    s[mt][0] = s[mt][1] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      s[mt][0] = Matrix<T>::mad(k[0][kk], q[mt][kk], s[mt][0]);
      s[mt][1] = Matrix<T>::mad(k[1][kk], q[mt][kk], s[mt][1]);
    }
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    if constexpr (!ALL) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[mt][i / 4][i % 4] = (seen[mt] >> i) & 1 ? s[mt][i / 4][i % 4] : -INFINITY;
    }
    most[mt] = s[mt][0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) most[mt] = fmaxf(most[mt], s[mt][i / 4][i % 4]);
    behind = behind || most[mt] > r.limit[mt];
  }
  if (__any(behind)) {
    bool huge = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float next = fmaxf(r.top[mt], row_max(most[mt]));
      const float less = r.top[mt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((r.top[mt] - next) * scale_log2);
      r.top[mt] = next;
      r.limit[mt] = next + kSlack / scale_log2;
      r.from[mt] = next == -INFINITY ? kLift : __builtin_fmaf(-next, scale_log2, kLift);
      huge = huge || (next != -INFINITY && __builtin_fabsf(next) > 1e38f);
      r.sum[mt] *= less;
#pragma unroll
      for (int j = 0; j < DV; ++j) r.o[mt][j] *= less;
    }
    r.huge = __any(huge);
  }
  if (r.huge) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        s[mt][i / 4][i % 4] = r.top[mt] == -INFINITY ? -INFINITY : (s[mt][i / 4][i % 4] - r.top[mt]) * scale_log2 + kLift;
  } else {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[mt][i / 4][i % 4] = __builtin_fmaf(s[mt][i / 4][i % 4], scale_log2, r.from[mt]);
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(s[mt][i / 4][i % 4]);
    r.sum[mt] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
    for (int i = 0; i < 4; ++i) w[mt][i] = pack2<T>(x[2 * i], x[2 * i + 1]);
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

__device__ __forceinline__ Share share_of(const AttentionArgs& a, int slot) {
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
struct Lookup {
  int page;
  uint32_t token;
};
struct Place {
  int64_t k, v;
  bool there;
};
__device__ __forceinline__ Lookup ask(const AttentionArgs& a, const Share& s, int old_steps, int step) {
  Lookup l{s.b, (uint32_t)step * kAttTile + (threadIdx.x & (kAttTile - 1))};
  if (step >= old_steps) {
    l.token -= (uint32_t)old_steps * kAttTile;
  } else if (a.cache.table != nullptr) {
    l.page = a.cache.table[s.b * a.cache.table_stride + a.cache.by_page.of(min(l.token, (uint32_t)s.len - 1))];      // (a step of the context has a token)
  }
  return l;
}
__device__ __forceinline__ Place place_of(const AttentionArgs& a, const Share& s, int old_steps, int step, const Lookup& l) {
  Place p;
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

// The rows that see node t add their weights times those of its values that are no finite numbers; `from`: the 4 DV values that a lane has, value 4 DV g + j
// in o[j % DV][j / DV] (PLAIN) or 16 (j / 4) + 4 g + j % 4 in o[j / 4][j % 4].
template <typename T, int D, int MT, bool PLAIN>
__device__ __forceinline__ void add_odd_values(Rows<MT, D / 16>& r, const T* values, int t, const u32x4 (&w)[MT], const uint32_t (&seen)[MT]) {
  constexpr int DV = D / 16;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, lane_of = (t >> 3) * 16 + n, i = t & 7;
  typedef T two __attribute__((ext_vector_type(2)));
  float by[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const uint32_t word = __shfl(i < 4 ? (i < 2 ? w[mt][0] : w[mt][1]) : (i < 6 ? w[mt][2] : w[mt][3]), lane_of);
    const two both = __builtin_bit_cast(two, word);
    by[mt] = (__shfl(seen[mt], lane_of) >> i) & 1 ? (float)(i & 1 ? both[1] : both[0]) : 0.f;
  }
#pragma unroll
  for (int j = 0; j < 4 * DV; ++j) {
    const float value = (float)values[PLAIN ? 4 * DV * g + j : 16 * (j / 4) + 4 * g + j % 4];
    if (!__builtin_isfinite(value))
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        if (by[mt] != 0.f) r.o[mt][PLAIN ? j % DV : j / 4][PLAIN ? j / DV : j % 4] += by[mt] * value;
  }
}

// The kernel for few rows.  One workgroup: up to 16 * MT rows (node, query head of one kv head) of one sequence over one part of its tokens; its wavefronts
// take steps of 32 tokens in turns and meet at the end.  K and V go from memory to the registers they are used from: K as it lies is an operand,
// V is loaded as it lies, D / 16 elements of 8 tokens to a lane, and turned inside the lane, 16 bits at a time.
// The weights are rounded to the type of V for the value product (their sum is not): half a step of each, so the error is a mean of independent
// roundings, below the one rounding of the result.
template <typename T, int D, int MT>
__global__ void __launch_bounds__(kAttWaves * 64, D <= 128 ? 2 : 1) tree_attention_kernel(const AttentionArgs a) {
  constexpr int KK = D / 32, DV = D / 16, N = DV / 2, R = 16 * MT;
  __shared__ float sums[kAttWaves][4 * DV * MT][64];
  __shared__ float2 tops[kAttWaves][MT][16];
  __shared__ __align__(16) int64_t places[kAttWaves][2][2][kAttTile];      // [..][turn][keys, values][token]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
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
  int step = share.first + wave, turn = 0;
  Lookup next{};
  if (step < last) next = ask(a, share, old_steps, step);
  load_queries<D, MT>(a, b, h, row_tile * R, q, node);
  Rows<MT, DV> rows;
  rows.clear(Matrix<T>::kLift);
  const int k_token = 8 * (n >> 2) + (n & 3);      // of the first 16; the second are 4 further
  const char *cache_k = a.cache.k + 2 * h * a.cache.head_stride, *cache_v = a.cache.v + 2 * h * a.cache.head_stride;
  const char *new_k = a.k_new.data + 2 * (b * a.k_new.batch_stride + h * a.k_new.head_stride),
             *new_v = a.v_new.data + 2 * (b * a.v_new.batch_stride + h * a.v_new.head_stride);

  for (; step < last; step += kAttWaves, turn ^= 1) {
    // The places pass through LDS, from the lane that looked one up to those that load from it.  A wavefront's own accesses there are in order.
    const bool old = step < old_steps;
    const Place mine = place_of(a, share, old_steps, step, next);
    int64_t(*table)[kAttTile] = places[wave][turn];
    if (lane < kAttTile) {
      table[0][lane] = mine.k;
      table[1][lane] = mine.v;
    }
    const uint32_t there = (uint32_t)__ballot(mine.there);
    const bool all = old && there == 0xffffffffu;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    u32x4 k[2][KK], w[MT];
    Words<N> v[8];
    const char *base_k = (old ? cache_k : new_k) + 16 * g, *base_v = (old ? cache_v : new_v) + 2 * DV * n;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const char* p = base_k + table[0][k_token + 4 * half];
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) k[half][kk] = *reinterpret_cast<const u32x4*>(p + 64 * kk);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = load_words<N>(base_v + table[1][8 * g + i]);
    if (step + kAttWaves < last) next = ask(a, share, old_steps, step + kAttWaves);
    uint32_t seen[MT] = {};
    if (all) {
      weigh<T, D, MT, true>(rows, q, k, a.scale_log2, seen, w);
    } else {
      const int t0 = (step - old_steps) * kAttTile;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        seen[mt] = (there >> (8 * g)) & 0xffu;
        if (!old) seen[mt] &= seen_of(a, b, node[mt], t0 + 8 * g);
      }
      weigh<T, D, MT, false>(rows, q, k, a.scale_log2, seen, w);
      // A token that is not there was read from a place that is, and counts as zeros.  A node may be seen by some rows only, and for the others its values may be
      // anything: what is no finite number leaves the product, in which it would meet weights of zero, and is added to the rows that see it by itself.
      bool odd = false;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const uint32_t is = (there >> (8 * g + i)) & 1 ? v[i].w[j] : 0u, number = old ? is : numbers<T>(is);
          odd = odd || number != is;
          v[i].w[j] = number;
        }
      if (__any(odd)) {
#pragma unroll 1
        for (int t = 0; t < min(kAttTile, a.seen_nodes - t0); ++t)
          add_odd_values<T, D, MT, true>(rows, reinterpret_cast<const T*>(new_v) + (t0 + t) * a.v_new.token_stride, t, w, seen);
      }
    }
#pragma unroll
    for (int j = 0; j < DV; ++j) {
      u32x4 t;
#pragma unroll
      for (int i = 0; i < 4; ++i) t[i] = __builtin_amdgcn_perm(v[2 * i + 1].w[j / 2], v[2 * i].w[j / 2], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) rows.o[mt][j] = Matrix<T>::mad(t, w[mt], rows.o[mt][j]);
    }
  }

  // the wavefronts' rows meet: each wavefront adds up the quarter 4 g + wave of the elements
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
    float m = -INFINITY, s = 0.f, f[kAttWaves];
#pragma unroll
    for (int w = 0; w < kAttWaves; ++w) m = fmaxf(m, tops[w][mt][n].x);
#pragma unroll
    for (int w = 0; w < kAttWaves; ++w) {
      f[w] = tops[w][mt][n].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((tops[w][mt][n].x - m) * a.scale_log2);
      s += tops[w][mt][n].y * f[w];
    }
    float e[DV];
#pragma unroll
    for (int j = 0; j < DV; ++j) {
      e[j] = 0.f;
#pragma unroll
      for (int w = 0; w < kAttWaves; ++w) e[j] += sums[w][(mt * 4 + wave) * DV + j][lane] * f[w];
    }
    if (r >= a.rows) continue;
    const int d = DV * (4 * g + wave);
    if (share.parts == 1) {
      const float by = m == -INFINITY ? 0.f : 1.f / s;
      uint32_t words[N];
#pragma unroll
      for (int j = 0; j < N; ++j) words[j] = pack2<T>(e[2 * j] * by, e[2 * j + 1] * by);
      const int head = h * a.group + r - node[mt] * a.group;
      store_words(a.out.data + 2 * (b * a.out.batch_stride + node[mt] * a.out.token_stride + head * a.out.head_stride + d), words);
      if (a.lse != nullptr && g == 0 && wave == 0) a.lse[((int64_t)b * a.nodes + node[mt]) * (a.kv_heads * a.group) + head] = log_sum<T>(m, s, a.scale);
    } else {
      const int64_t row = part_row(a, slot, h, row_tile, R) + mt * 16 + n;
      uint32_t words[DV];
#pragma unroll
      for (int j = 0; j < DV; ++j) words[j] = __builtin_bit_cast(uint32_t, e[j]);
      if (m != -INFINITY) store_words(reinterpret_cast<char*>(a.part + row * D + d), words);
      if (g == 0 && wave == 0) a.stats[row] = make_float2(m, s);
    }
  }
}

// The parts of a row meet: one wavefront to a row.  Tops first, then sums of eight parts at a time, so that their loads are on the way together.
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
  const float by = m == -INFINITY ? 0.f : 1.f / s;
  const int node = a.by_group.of(r), head = h * a.group + r - node * a.group;
  char* out = a.out.data + 2 * (b * a.out.batch_stride + node * a.out.token_stride + head * a.out.head_stride + at);
  if (D >= 128 || lane < D / 2)
#pragma unroll
    for (int j = 0; j < P; ++j) *reinterpret_cast<uint32_t*>(out + 256 * j) = pack2<T>(e[2 * j] * by, e[2 * j + 1] * by);
  if (a.lse != nullptr && lane == 0) a.lse[((int64_t)b * a.nodes + node) * (a.kv_heads * a.group) + head] = log_sum<T>(m, s, a.scale);
}

// The kernel for many rows: WAVES wavefronts with 16 * MT rows each take every step together.  K and V of a step are loaded once for all of them and kept
// in LDS, two steps in turns: the next step's are asked for before this one's products and written behind them, and the places of the tokens
// of the step after that are looked up meanwhile.
//   K: pieces of 8 elements [D / 8][32 tokens], the tokens' places exclusive-or the piece's number, so that neither the writing (a row of the
//      cache at a time) nor the reading (16 tokens of four pieces) meets itself in a bank;
//   V: turned while it is written: [4 groups of 8 tokens][D] of 16 bytes, as the value product reads it.
// A lane's results are the values 16 j + 4 g ... + 3 of its row, j < D / 16.
template <typename T, int D, int MT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, D <= 128 ? 2 : 1) tree_attention_wide_kernel(const AttentionArgs a) {
  constexpr int KK = D / 32, DV = D / 16, R = 16 * MT * WAVES, THREADS = WAVES * 64;
  constexpr int U = (4 * D + THREADS - 1) / THREADS;      // units of 16 bytes of K, and of V, to a thread
  __shared__ __align__(16) char lds_k[2][4 * D * 16], lds_v[2][4 * D * 16];
  __shared__ __align__(16) int64_t places[2][2][kAttTile];      // [step % 2][keys, values][token]
  __shared__ uint32_t lds_there[4], lds_odd[2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  uint32_t id = blockIdx.x;
  const int h = id % a.kv_heads;
  id /= a.kv_heads;
  const int row_tile = id % a.row_tiles, slot = id / a.row_tiles;
  const Share share = share_of(a, slot);
  if (share.b < 0) return;
  const int b = share.b, old_steps = steps_of(share.len), first = share.first, last = share.last;
  if (share.part == 0 && h == 0 && row_tile == 0 && threadIdx.x == 0 && a.places != nullptr) a.places[b] = make_int2(slot, share.parts);

  // The first wavefront looks places up; those of step s are in places[s % 2] from the barrier two steps before its products on.
  auto keep_places = [&](int step, const Lookup& l) {
    const Place mine = place_of(a, share, old_steps, step, l);
    if (lane < kAttTile) {
      places[step & 1][0][lane] = mine.k;
      places[step & 1][1][lane] = mine.v;
    }
    const uint32_t there = (uint32_t)__ballot(mine.there);
    if (lane == 0) lds_there[step & 3] = there;
  };
  if (wave == 0) {
    if (first < last) keep_places(first, ask(a, share, old_steps, first));
    if (first + 1 < last) keep_places(first + 1, ask(a, share, old_steps, first + 1));
  }
  if (threadIdx.x < 2) lds_odd[threadIdx.x] = 0;
  u32x4 q[MT][KK];
  int node[MT];
  load_queries<D, MT>(a, b, h, row_tile * R + wave * 16 * MT, q, node);
  const bool works = row_tile * R + wave * 16 * MT < a.rows;      // a wavefront without rows only loads
  Rows<MT, DV> rows;
  rows.clear(Matrix<T>::kLift);

  // What this thread loads of a step: unit u of K is piece u % (D / 8) of token u / (D / 8); of V it is the elements 2 (u % (D / 2)) and the next of four tokens.
  const char *cache_k = a.cache.k + 2 * h * a.cache.head_stride, *cache_v = a.cache.v + 2 * h * a.cache.head_stride;
  const char *new_k = a.k_new.data + 2 * (b * a.k_new.batch_stride + h * a.k_new.head_stride),
             *new_v = a.v_new.data + 2 * (b * a.v_new.batch_stride + h * a.v_new.head_stride);
  u32x4 load_k[U];
  uint32_t load_v[U][4];
  auto load = [&](int step) {
    const bool old = step < old_steps;
    const char *base_k = old ? cache_k : new_k, *base_v = old ? cache_v : new_v;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = min((int)threadIdx.x + i * THREADS, 4 * D - 1);
      load_k[i] = *reinterpret_cast<const u32x4*>(base_k + places[step & 1][0][u / (D / 8)] + 16 * (u % (D / 8)));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        load_v[i][j] = *reinterpret_cast<const uint32_t*>(base_v + places[step & 1][1][4 * (u / (D / 2)) + j] + 4 * (u % (D / 2)));
    }
  };
  auto keep = [&](int step, int buffer) {
    const uint32_t there = lds_there[step & 3];
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
          const uint32_t is = (there >> (4 * four + j)) & 1 ? load_v[i][j] : 0u, number = old ? is : numbers<T>(is);
          odd = odd || number != is;
          load_v[i][j] = number;
        }
      }
      const int token = u / (D / 8), place = ((token >> 2) & 1) * 16 + 4 * (token >> 3) + (token & 3);      // as weigh() numbers the tokens
      const int piece = u % (D / 8);
      *reinterpret_cast<u32x4*>(lds_k[buffer] + (piece * kAttTile + (place ^ (piece & 15))) * 16) = load_k[i];
      char* to = lds_v[buffer] + ((four >> 1) * D + d) * 16 + (four & 1) * 8;
      const uint32_t* v = load_v[i];
      *reinterpret_cast<uint2*>(to) = make_uint2(__builtin_amdgcn_perm(v[1], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[2], 0x05040100u));
      *reinterpret_cast<uint2*>(to + 16) = make_uint2(__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u));
    }
    if (odd) lds_odd[buffer] = step + 1;      // of this step; whatever else stands there is another's
  };

  __syncthreads();
  if (first < last) {
    load(first);
    keep(first, 0);
  }
  __syncthreads();
  for (int step = first; step < last; ++step) {
    const int buffer = (step - first) & 1;
    Lookup after{};
    if (wave == 0 && step + 2 < last) after = ask(a, share, old_steps, step + 2);
    if (step + 1 < last) load(step + 1);
    if (works) {
      const uint32_t there = lds_there[step & 3];
      const bool old = step < old_steps;
      u32x4 k[2][KK], w[MT];
      uint32_t seen[MT] = {};
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) k[half][kk] = *reinterpret_cast<const u32x4*>(lds_k[buffer] + ((4 * kk + g) * kAttTile + half * 16 + (n ^ ((4 * kk + g) & 15))) * 16);
      if (old && there == 0xffffffffu) {
        weigh<T, D, MT, true>(rows, q, k, a.scale_log2, seen, w);
      } else {
        const int t0 = (step - old_steps) * kAttTile;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          seen[mt] = (there >> (8 * g)) & 0xffu;
          if (!old) seen[mt] &= seen_of(a, b, node[mt], t0 + 8 * g);
        }
        weigh<T, D, MT, false>(rows, q, k, a.scale_log2, seen, w);
        if (!old && lds_odd[buffer] == (uint32_t)step + 1) {
#pragma unroll 1
          for (int t = 0; t < min(kAttTile, a.seen_nodes - t0); ++t)
            add_odd_values<T, D, MT, false>(rows, reinterpret_cast<const T*>(new_v) + (t0 + t) * a.v_new.token_stride, t, w, seen);
        }
      }
#pragma unroll
      for (int j = 0; j < DV; ++j) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(lds_v[buffer] + (g * D + 16 * j + n) * 16);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) rows.o[mt][j] = Matrix<T>::mad(v, w[mt], rows.o[mt][j]);
      }
    }
    if (step + 1 < last) keep(step + 1, buffer ^ 1);
    if (wave == 0 && step + 2 < last) keep_places(step + 2, after);      // over those of this step, which were read before the last barrier
    __syncthreads();
  }
  if (!works) return;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int in_tile = wave * 16 * MT + mt * 16 + n, r = row_tile * R + in_tile;
    float s = rows.sum[mt];
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (r >= a.rows) continue;
    const float m = rows.top[mt];
    if (share.parts == 1) {
      const float by = m == -INFINITY ? 0.f : 1.f / s;
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
