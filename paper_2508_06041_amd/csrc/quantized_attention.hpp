// Attention of new tokens (the nodes of a tree, a chain, one) over a cache that holds keys and values in 8 or 4 bits, and over one another.
//
// With key codes c, their scale s (and offset f) the score of a cached token is x = s (q . c) + f (sum of q), and with value codes d, scale u (and offset g) its part of the
// result is w u d + w g.  So the codes go into the matrix pipe as they are, whole or half numbers that 16 bits hold exactly, and scales and offsets
// meet scores and weights in 32 bits: no value is rounded that was not rounded when it was quantised.  The weights w u are rounded to bfloat16, whose range is that of a float, for bfloat16
// results; for float16 ones they go in as two such numbers, w u and what is left of it, which is 16 bits of precision for twice the value products.
#pragma once
#include <type_traits>

#include "quantized_cache.hpp"
#include "tree_attention.hpp"

namespace dpllm {

struct QuantizedArgs : AttentionArgs {      // cache: codes, strides in bytes
  const uint32_t *k_scales, *v_scales;      // of the layer; strides in words
  int64_t scale_page, scale_token, scale_head;
};

template <int FORMAT, int D>
struct Held {
  static constexpr int DV = D / 16;                      // dimensions of the values to a lane
  static constexpr int BITS = FORMAT == kInt4 ? 4 : 8;
  static constexpr int KW = D * BITS / 128;              // words of a key to a lane: a quarter of it
  static constexpr int VW = (DV * BITS + 31) / 32;       // words of a value to a lane
};

// Dimension j of the values that lane n of sixteen holds.  Six to a lane are four and two, so that both are read at their alignment.
template <int D>
__device__ __forceinline__ constexpr int value_dim(int n, int j) {
  return D == 96 ? (j < 4 ? 4 * n + j : 64 + 2 * n + j - 4) : D / 16 * n + j;
}

template <int N>
struct Codes {
  uint32_t w[N];
};

// A quarter of a key's codes from p on (N words; 16-byte aligned where N is a multiple of 4).
template <int N>
__device__ __forceinline__ Codes<N> load_codes(const char* p) {
  const Words<N> r = load_words<N>(p);
  Codes<N> c;
#pragma unroll
  for (int i = 0; i < N; ++i) c.w[i] = r.w[i];
  return c;
}

// Lane n's codes of a value that starts at p.
template <int FORMAT, int D>
__device__ __forceinline__ Codes<Held<FORMAT, D>::VW> load_value(const char* p, int n) {
  Codes<Held<FORMAT, D>::VW> c;
  if constexpr (D == 96 && FORMAT == kInt4) {
    c.w[0] = *reinterpret_cast<const uint16_t*>(p + 2 * n) | (uint32_t) * reinterpret_cast<const uint8_t*>(p + 32 + n) << 16;
  } else if constexpr (D == 96) {
    c.w[0] = *reinterpret_cast<const uint32_t*>(p + 4 * n);
    c.w[1] = *reinterpret_cast<const uint16_t*>(p + 64 + 2 * n);
  } else if constexpr (D == 64 && FORMAT == kInt4) {
    c.w[0] = *reinterpret_cast<const uint16_t*>(p + 2 * n);
  } else {
    c = load_codes<Held<FORMAT, D>::VW>(p + 4 * Held<FORMAT, D>::VW * n);
  }
  return c;
}

// Eight elements of a query or a node's key in the order in which the codes of eight come out of key_operand.
template <int FORMAT>
__device__ __forceinline__ u32x4 in_code_order(u32x4 x) {
  if constexpr (FORMAT != kInt4) return x;
  return u32x4{__builtin_amdgcn_perm(x[1], x[0], 0x05040100u), __builtin_amdgcn_perm(x[3], x[2], 0x05040100u), __builtin_amdgcn_perm(x[1], x[0], 0x07060302u),
               __builtin_amdgcn_perm(x[3], x[2], 0x07060302u)};      // 0 2, 4 6, 1 3, 5 7
}
// Codes 8 kk ... + 7 of a lane's quarter of a key.
template <int FORMAT, typename T, int N>
__device__ __forceinline__ u32x4 key_operand(const Codes<N>& c, int kk) {
  if constexpr (FORMAT == kInt4) {
    const uint32_t even = level_bytes(c.w[kk]), odd = level_bytes(c.w[kk] >> 4);
    return u32x4{two_codes<FORMAT, T>(even, false), two_codes<FORMAT, T>(even, true), two_codes<FORMAT, T>(odd, false), two_codes<FORMAT, T>(odd, true)};
  } else {
    return u32x4{two_codes<FORMAT, T>(c.w[2 * kk], false), two_codes<FORMAT, T>(c.w[2 * kk], true), two_codes<FORMAT, T>(c.w[2 * kk + 1], false),
                 two_codes<FORMAT, T>(c.w[2 * kk + 1], true)};
  }
}
// Dimensions 0 ... DV - 1 of two tokens' values, a pair of bfloat16 for each.
template <int FORMAT, int DV, int N>
__device__ __forceinline__ void value_pairs(const Codes<N>& a, const Codes<N>& b, uint32_t (&pair)[DV]) {
  if constexpr (FORMAT == kInt4) {
#pragma unroll
    for (int w = 0; w < N; ++w)
#pragma unroll
      for (int odd = 0; odd < 2; ++odd) {
        const uint32_t x = level_bytes(a.w[w] >> (4 * odd)), y = level_bytes(b.w[w] >> (4 * odd));
        const uint32_t low = __builtin_amdgcn_perm(y, x, 0x05010400u), high = __builtin_amdgcn_perm(y, x, 0x07030602u);
        if (8 * w + odd < DV) pair[8 * w + odd] = two_codes<FORMAT, bfloat_t>(low, false);
        if (8 * w + odd + 2 < DV) pair[8 * w + odd + 2] = two_codes<FORMAT, bfloat_t>(low, true);
        if (8 * w + odd + 4 < DV) pair[8 * w + odd + 4] = two_codes<FORMAT, bfloat_t>(high, false);
        if (8 * w + odd + 6 < DV) pair[8 * w + odd + 6] = two_codes<FORMAT, bfloat_t>(high, true);
      }
  } else {
#pragma unroll
    for (int w = 0; w < N; ++w) {
      const uint32_t low = __builtin_amdgcn_perm(b.w[w], a.w[w], 0x05010400u), high = __builtin_amdgcn_perm(b.w[w], a.w[w], 0x07030602u);
      pair[4 * w] = two_codes<FORMAT, bfloat_t>(low, false);
      pair[4 * w + 1] = two_codes<FORMAT, bfloat_t>(low, true);
      if (4 * w + 2 < DV) pair[4 * w + 2] = two_codes<FORMAT, bfloat_t>(high, false);
      if (4 * w + 3 < DV) pair[4 * w + 3] = two_codes<FORMAT, bfloat_t>(high, true);
    }
  }
}

// Eight weights as bfloat16; with `rest`, that and what the rounding left of them.
__device__ __forceinline__ u32x4 rounded(const float (&w)[8]) {
  return u32x4{pack2<bfloat_t>(w[0], w[1]), pack2<bfloat_t>(w[2], w[3]), pack2<bfloat_t>(w[4], w[5]), pack2<bfloat_t>(w[6], w[7])};
}
__device__ __forceinline__ u32x4 rest_of(const float (&w)[8], const u32x4& r) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = w[i] - __uint_as_float(i & 1 ? r[i / 2] & 0xffff0000u : r[i / 2] << 16);
  return rounded(x);
}

// Where the 32 tokens of a step of the cache lie; as in tree_attention.hpp, but codes and scales have places of their own.
struct HeldPlace {
  int64_t at, scale_at;      // of a token that is not there: of one that is
  bool there;
};
__device__ __forceinline__ Lookup ask_held(const QuantizedArgs& a, const Share& s, int last, int step) {
  Lookup l{s.b, (uint32_t)step * kAttTile + (threadIdx.x & (kAttTile - 1))};
  if (step < last && a.cache.table != nullptr) l.page = a.cache.table[s.b * a.cache.table_stride + a.cache.by_page.of(min(l.token, (uint32_t)s.len - 1))];
  return l;
}
__device__ __forceinline__ HeldPlace held_place(const QuantizedArgs& a, const Share& s, int last, int step, const Lookup& l) {
  HeldPlace p{0, 0, false};
  if (step >= last) return p;
  p.there = l.token < (uint32_t)s.len && (uint32_t)l.page < (uint32_t)a.cache.pages;
  const int64_t in_page = (int64_t)(l.token - a.cache.by_page.of(l.token) * (uint32_t)a.cache.page);
  p.at = p.there ? l.page * a.cache.page_stride + in_page * a.cache.token_stride : 0;
  p.scale_at = p.there ? l.page * a.scale_page + in_page * a.scale_token : 0;
  return p;
}

// Queries in the order of a lane's quarter of a key: element 8 kk + e of lane group g is g D / 4 + 8 kk + e of the head.
template <int FORMAT, int D, int MT>
__device__ __forceinline__ void load_quarters(const QuantizedArgs& a, int b, int h, int first, u32x4 (&q)[MT][D / 32], int (&node)[MT]) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = first + mt * 16 + n;
    node[mt] = -1;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) q[mt][kk] = u32x4{0, 0, 0, 0};
    if (r < a.rows) {
      node[mt] = a.by_group.of(r);
      const char* p = a.q.data + 2 * (b * a.q.batch_stride + node[mt] * a.q.token_stride + (h * a.group + r - node[mt] * a.group) * a.q.head_stride + g * (D / 4));
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) q[mt][kk] = in_code_order<FORMAT>((*reinterpret_cast<const u32x4*>(p + 16 * kk) & a.keep) ^ a.sign);
    }
  }
}
// The sum of a row's query, for the offsets of the keys.
template <typename T, int D, int MT>
__device__ __forceinline__ void sum_queries(const u32x4 (&q)[MT][D / 32], float (&sum)[MT]) {
  typedef T two __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float s = 0.f;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const two v = __builtin_bit_cast(two, (uint32_t)q[mt][kk][i]);
        s += (float)v[0] + (float)v[1];
      }
    s += __shfl_xor(s, 16);
    sum[mt] = s + __shfl_xor(s, 32);
  }
}

// Scores of codes become scores of keys.  k: the words of the lane's eight tokens.
template <int FORMAT, int MT>
__device__ __forceinline__ void scale_scores(Scores<MT>& s, const uint32_t (&k)[8], const float (&q_sum)[MT]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float by = scale_of<FORMAT>(k[i]);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float x = s[mt][i / 4][i % 4];
      s[mt][i / 4][i % 4] = FORMAT == kInt4 ? __builtin_fmaf(x, by, offset_of(k[i]) * q_sum[mt]) : x * by;
    }
  }
}

// The kernel for few rows: as tree_attention_kernel, with steps of codes in front of those of the nodes.  A lane reads a quarter of each of two keys (16 to 64
// bytes in a row) and its dimensions of eight values; the next step's are on their way while this one's are used, as a step of codes has half or a quarter of the bytes
// in flight that one of numbers has.
template <int FORMAT, typename T, int D, int MT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, D <= 128 ? 2 : 1) quantized_attention_kernel(const QuantizedArgs a) {
  typedef Held<FORMAT, D> H;
  constexpr int KK = D / 32, DV = D / 16, R = 16 * MT;
  constexpr int PER = 4 * DV / WAVES;      // of a lane's 4 DV results, what a wavefront adds up in the end
  constexpr bool TWO = __is_same(T, half_t);
  __shared__ float sums[WAVES][4 * DV * MT][64];
  __shared__ float offsets[WAVES][MT][16];
  __shared__ float2 tops[WAVES][MT][16];
  __shared__ __align__(16) int64_t places[WAVES][2][kAttTile];
  __shared__ __align__(16) uint32_t words[WAVES][2][kAttTile];      // of keys, of values
  const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  uint32_t id = blockIdx.x;
  const int h = id % a.kv_heads;
  id /= a.kv_heads;
  const int row_tile = id % a.row_tiles, slot = id / a.row_tiles;
  const Share share = share_of(a, slot);
  if (share.b < 0) return;
  const int b = share.b, old_steps = steps_of(share.len), last = share.last, last_old = min(last, old_steps);
  if (share.part == 0 && h == 0 && row_tile == 0 && threadIdx.x == 0 && a.places != nullptr) a.places[b] = make_int2(slot, share.parts);

  u32x4 q[MT][KK];
  float q_sum[MT] = {}, offset[MT] = {};
  int node[MT];
  int step = share.first + wave;
  Lookup next = ask_held(a, share, last_old, step);
  load_quarters<FORMAT, D, MT>(a, b, h, row_tile * R, q, node);
  if (FORMAT == kInt4) sum_queries<T, D, MT>(q, q_sum);
  Rows<MT, DV> rows;
  rows.clear();
  const int k_token = 8 * (n >> 2) + (n & 3);      // of the first 16; the second are 4 further
  const char *cache_k = a.cache.k + h * a.cache.head_stride, *cache_v = a.cache.v + h * a.cache.head_stride;
  const uint32_t* scales = (lane < kAttTile ? a.k_scales : a.v_scales) + h * a.scale_head;
  struct Tokens {
    Codes<H::KW> k[2];
    Codes<H::VW> v[8];
    uint32_t word, there;
  };
  auto load = [&](int step, int turn, Tokens& x) {
    const HeldPlace mine = held_place(a, share, last_old, step, next);
    x.word = scales[mine.scale_at];
    if (!mine.there) x.word = 0u;
    if (lane < kAttTile) places[wave][turn][lane] = mine.at;
    x.there = (uint32_t)__ballot(mine.there);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int half = 0; half < 2; ++half) x.k[half] = load_codes<H::KW>(cache_k + places[wave][turn][k_token + 4 * half] + g * (D * H::BITS / 32));
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i] = load_value<FORMAT, D>(cache_v + places[wave][turn][8 * g + i], n);
    next = ask_held(a, share, last_old, step + WAVES);
  };
  // The sums of offsets are relative to the rows' tops too.
  auto follow = [&](const float (&before)[MT]) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
      if (rows.top[mt] != before[mt]) offset[mt] *= before[mt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((before[mt] - rows.top[mt]) * a.scale_log2);
  };
  auto attend = [&](Tokens& x) {
    const bool all = x.there == 0xffffffffu;
    words[wave][lane >> 5][lane & 31] = x.word;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    uint32_t k_word[8], v_word[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 p = *reinterpret_cast<const u32x4*>(&words[wave][0][8 * g + 4 * i]), r = *reinterpret_cast<const u32x4*>(&words[wave][1][8 * g + 4 * i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        k_word[4 * i + j] = p[j];
        v_word[4 * i + j] = r[j];
      }
    }
    u32x4 k[2][KK];
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) k[half][kk] = key_operand<FORMAT, T>(x.k[half], kk);
    Scores<MT> s;
    score<T, D, MT>(q, k, s);
    scale_scores<FORMAT, MT>(s, k_word, q_sum);
    if (!all) {
      uint32_t seen[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) seen[mt] = (x.there >> (8 * g)) & 0xffu;
      mask<MT>(s, seen);
      // a token that is not there was read from a place that is, and counts as zeros
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < H::VW; ++j) x.v[i].w[j] = (x.there >> (8 * g + i)) & 1 ? x.v[i].w[j] : 0u;
    }
    Weights w[MT];
    float before[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) before[mt] = rows.top[mt];
    weigh<T, MT, DV>(rows, s, a.scale_log2, w);
    if (FORMAT == kInt4) follow(before);
    u32x4 p[MT], rest[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (FORMAT == kInt4)
#pragma unroll
        for (int i = 0; i < 8; ++i) offset[mt] = __builtin_fmaf(w[mt].w[i], offset_of(v_word[i]), offset[mt]);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[mt].w[i] *= scale_of<FORMAT>(v_word[i]);
      p[mt] = rounded(w[mt].w);
      if (TWO) rest[mt] = rest_of(w[mt].w, p[mt]);
    }
    uint32_t pairs[4][DV];
#pragma unroll
    for (int i = 0; i < 4; ++i) value_pairs<FORMAT, DV>(x.v[2 * i], x.v[2 * i + 1], pairs[i]);
#pragma unroll
    for (int j = 0; j < DV; ++j) {
      const u32x4 t{pairs[0][j], pairs[1][j], pairs[2][j], pairs[3][j]};
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        rows.o[mt][j] = Matrix<bfloat_t>::mad(t, p[mt], rows.o[mt][j]);
        if (TWO) rows.o[mt][j] = Matrix<bfloat_t>::mad(t, rest[mt], rows.o[mt][j]);
      }
    }
  };
  if (step < last_old) {
    Tokens x, y;
    load(step, 0, x);
    for (; step < last_old; step += 2 * WAVES) {
      load(step + WAVES, 1, y);
      attend(x);
      if (step + WAVES >= last_old) {
        step += WAVES;
        break;
      }
      load(step + 2 * WAVES, 0, x);
      attend(y);
    }
  }

  // the nodes, as they are
  const char *new_k = a.k_new.data + 2 * (b * a.k_new.batch_stride + h * a.k_new.head_stride),
             *new_v = a.v_new.data + 2 * (b * a.v_new.batch_stride + h * a.v_new.head_stride);
  bool odd = false;      // among the values is something that is no finite number
  for (; step < last; step += WAVES) {
    const int t0 = (step - old_steps) * kAttTile, here = a.seen_nodes - t0;
    u32x4 k[2][KK], w[MT];
    Scores<MT> s;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int t = k_token + 4 * half;
      const char* p = new_k + 2 * ((t < here ? t0 + t : 0) * a.k_new.token_stride + g * (D / 4));
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) k[half][kk] = in_code_order<FORMAT>(*reinterpret_cast<const u32x4*>(p + 16 * kk));
    }
    uint32_t v[8][DV / 2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool there = 8 * g + i < here;
      const char* p = new_v + 2 * (there ? t0 + 8 * g + i : 0) * a.v_new.token_stride;
#pragma unroll
      for (int j = 0; j < DV / 2; ++j) {
        const uint32_t is = there ? *reinterpret_cast<const uint32_t*>(p + 2 * value_dim<D>(n, 2 * j)) : 0u, number = numbers<T>(is);
        odd = odd || number != is;
        v[i][j] = number;
      }
    }
    score<T, D, MT>(q, k, s);
    uint32_t seen[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) seen[mt] = seen_of(a, b, node[mt], t0 + 8 * g) & (here - 8 * g >= 8 ? 0xffu : here > 8 * g ? (1u << (here - 8 * g)) - 1u : 0u);
    mask<MT>(s, seen);
    float before[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) before[mt] = rows.top[mt];
    weigh<T, MT, DV>(rows, s, a.scale_log2, w);
    if (FORMAT == kInt4) follow(before);
#pragma unroll
    for (int j = 0; j < DV; ++j) {
      u32x4 t;
#pragma unroll
      for (int i = 0; i < 4; ++i) t[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) rows.o[mt][j] = Matrix<T>::mad(t, w[mt], rows.o[mt][j]);
    }
  }
  if (__any(odd)) {      // a value above a weight of zero is left out; a weight above zero changes no infinity and no NaN
#pragma unroll 1
    for (int t = max(share.first - old_steps, 0) * kAttTile; t < min((last - old_steps) * kAttTile, a.seen_nodes); ++t) {
      if ((old_steps + t / kAttTile - share.first) % WAVES != wave) continue;
      const T* values = reinterpret_cast<const T*>(new_v) + t * a.v_new.token_stride;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < DV; ++j) {
          const float value = (float)values[value_dim<D>(4 * g + i, j)];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
            if (((seen_of(a, b, node[mt], t & ~7) >> (t & 7)) & 1) && !__builtin_isfinite(value)) rows.o[mt][j][i] += value;
        }
    }
  }

  // the wavefronts' rows meet: each wavefront adds up its part of the elements
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float s = rows.sum[mt];
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    float f = offset[mt];
    if (FORMAT == kInt4) {
      f += __shfl_xor(f, 16);
      f += __shfl_xor(f, 32);
    }
    if (g == 0) {
      tops[wave][mt][n] = make_float2(rows.top[mt], s);
      offsets[wave][mt][n] = f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < DV; ++j) sums[wave][(mt * 4 + i) * DV + j][lane] = rows.o[mt][j][i];
  }
  __syncthreads();
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = row_tile * R + mt * 16 + n;
    float m = -INFINITY, s = 0.f, f[WAVES], plus = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, tops[w][mt][n].x);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      f[w] = tops[w][mt][n].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((tops[w][mt][n].x - m) * a.scale_log2);
      s += tops[w][mt][n].y * f[w];
      if (FORMAT == kInt4) plus += offsets[w][mt][n] * f[w];
    }
    float e[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      e[j] = plus;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) e[j] += sums[w][mt * 4 * DV + wave * PER + j][lane] * f[w];
    }
    if (r >= a.rows) continue;
    const bool whole = share.parts == 1;
    const int head = h * a.group + r - node[mt] * a.group;
    const float by = one_over(s);
    char* out = a.out.data + 2 * (b * a.out.batch_stride + node[mt] * a.out.token_stride + head * a.out.head_stride);
    const int64_t row = part_row(a, slot, h, row_tile, R) + mt * 16 + n;
    // the elements wave * PER ... of [4][DV], in runs that lie side by side
    auto put = [&](auto length, int from) {
      constexpr int L = decltype(length)::value;
      const int d = value_dim<D>(4 * g + (wave * PER + from) / DV, (wave * PER + from) % DV);
      if (whole) {
        uint32_t w[L / 2];
#pragma unroll
        for (int j = 0; j < L / 2; ++j) w[j] = pack2<T>(e[from + 2 * j] * by, e[from + 2 * j + 1] * by);
        store_words(out + 2 * d, w);
      } else if (m != -INFINITY) {
        uint32_t w[L];
#pragma unroll
        for (int j = 0; j < L; ++j) w[j] = __builtin_bit_cast(uint32_t, e[from + j]);
        store_words(reinterpret_cast<char*>(a.part + row * D + d), w);
      }
    };
    if constexpr (D == 96) {
      put(std::integral_constant<int, 4>(), 0);
      put(std::integral_constant<int, 2>(), 4);
    } else {
      put(std::integral_constant<int, PER>(), 0);
    }
    if (g == 0 && wave == 0) {
      if (!whole)
        a.stats[row] = make_float2(m, s);
      else if (a.lse != nullptr)
        a.lse[((int64_t)b * a.nodes + node[mt]) * (a.kv_heads * a.group) + head] = log_sum<T>(m, s, a.scale);
    }
  }
}

}  // namespace dpllm
