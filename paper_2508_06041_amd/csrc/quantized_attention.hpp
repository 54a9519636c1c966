// Attention of new tokens (the nodes of a tree, a chain, one) over a cache that holds keys and values in 8 or 4 bits, and over one another.
//
// With key codes c, their scale s (and offset f) the score of a cached token is x = s (q . c) + f (sum of q), and with value codes d, scale u (and offset g) its part of the
// result is w u d + w g.  So the codes go into the matrix pipe as they are, whole or half numbers that 16 bits hold exactly, and scales and offsets
// meet scores and weights in 32 bits: no value is rounded that was not rounded when it was quantised.  Codes are exact in bfloat16, which has the range of a float, so the weights w u go there as they
// are however far the scales of tokens lie apart, in two parts (the second is what rounding the first leaves): 16 bits of them, an error of 2^-16, which is little beside the rounding of either type's results.
// (In float16 they would have to be relative to a common unit, beside which the weights of tokens of small values vanish.)  Results of bfloat16 took less with one part in float16: for up to 16 rows nothing in
// 8 bits and 5 % in INT4, for 52 rows 5 to 7 %, in the kernel for many rows 10 to 20 % (100 rows over 9000 to 65001 tokens 126 us instead of 143 in e4m3, 142 instead of 157 in INT4); but they were off by up to a
// step more.
#pragma once
#include "quantized_cache.hpp"
#include "tree_attention.hpp"

namespace dpllm {

struct QuantizedArgs : AttentionArgs {      // cache: codes, strides in bytes
  const uint32_t *k_scales, *v_scales;      // of the layer; strides in words
  int64_t scale_page, scale_token, scale_head;
  int heads_at_once, turns;                 // wavefronts of a workgroup: heads x turns
};

template <int FORMAT, int D>
struct Held {
  static constexpr int DV = D / 16;                      // dimensions of the values to a lane
  static constexpr int BITS = FORMAT == kInt4 ? 4 : 8;
  static constexpr int KW = D * BITS / 128;              // words of a key to a lane: a quarter of it
  static constexpr int VW = (DV * BITS + 31) / 32;       // words of a value to a lane
  static constexpr int BYTES = D * BITS / 8;             // of a key or value
  static constexpr int PIECES = BYTES / 16;
  static constexpr int ROW = PIECES % 2 ? BYTES : BYTES + 16;      // in LDS: an odd number of pieces, so that sixteen rows are in as many banks
  static constexpr int LOADS = (32 * PIECES + 63) / 64;  // pieces of 32 keys to a lane
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

// 16 bytes of a token.  Heads that fill whole lines of 128 bytes are read once and need not stay in the caches (400000 tokens of 8 heads of 128 e4m3 codes, 845 MB: 159 us with them,
// 139 past them); others share their lines with a neighbour, which is to find them there (heads of 64: 95 us against 102 past them, in 4 bits 82 against 94).
template <bool ONCE>
__device__ __forceinline__ u32x4 load_piece(const char* p) {
  const u32x4* at = reinterpret_cast<const u32x4*>(p);
  if constexpr (ONCE) return __builtin_nontemporal_load(at);
  return *at;
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
    const uint32_t even = level_bytes<false>(c.w[kk]), odd = level_bytes<true>(c.w[kk]);
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
    auto half = [&](int first, uint32_t x, uint32_t y) {      // dimensions first, first + 2, ...
      const uint32_t low = __builtin_amdgcn_perm(y, x, 0x05010400u), high = __builtin_amdgcn_perm(y, x, 0x07030602u);
      if (first < DV) pair[first] = two_codes<FORMAT, bfloat_t>(low, false);
      if (first + 2 < DV) pair[first + 2] = two_codes<FORMAT, bfloat_t>(low, true);
      if (first + 4 < DV) pair[first + 4] = two_codes<FORMAT, bfloat_t>(high, false);
      if (first + 6 < DV) pair[first + 6] = two_codes<FORMAT, bfloat_t>(high, true);
    };
#pragma unroll
    for (int w = 0; w < N; ++w) {
      half(8 * w, level_bytes<false>(a.w[w]), level_bytes<false>(b.w[w]));
      half(8 * w + 1, level_bytes<true>(a.w[w]), level_bytes<true>(b.w[w]));
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

// Workgroups go to the eight parts of the chip in turns, and each part has a cache of its own with lines of 128 bytes, which hold one head of a token, or two.  So the heads
// (and tiles of rows) of a slot are on the same part, next to one another: a token's heads are read together, and no line twice.
// Of the heads, `heads` are taken by a workgroup.
__device__ __forceinline__ void place_group(const QuantizedArgs& a, int heads, int& slot, int& h, int& row_tile) {
  const uint32_t sets = (uint32_t)(a.kv_heads / heads), tiles = sets * a.row_tiles, even = (uint32_t)a.slots / 8 * 8;
  uint32_t t;
  if (blockIdx.x < even * tiles) {
    const uint32_t j = blockIdx.x >> 3;
    slot = (int)(j / tiles * 8 + (blockIdx.x & 7));
    t = j % tiles;
  } else {
    const uint32_t j = blockIdx.x - even * tiles;
    slot = (int)(even + j / tiles);
    t = j % tiles;
  }
  h = (int)(t % sets) * heads;
  row_tile = (int)(t / sets);
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

// Two numbers as T, into word i of p, and what that leaves of them into that of rest.
template <typename T>
__device__ __forceinline__ void two_parts(float a, float b, u32x4& p, u32x4& rest, int i) {
  typedef T two __attribute__((ext_vector_type(2)));
  uint32_t both = pack2<T>(a, b);      // (__builtin_bit_cast of a vector's element takes its first)
  p[i] = both;
  asm("" : "+v"(both));      // (else each half is made once more)
  const two h = __builtin_bit_cast(two, both);
  rest[i] = pack2<T>(a - (float)h[0], b - (float)h[1]);
}

// The weights of a step from the products of codes, with the scales (and offsets) of the lane's eight tokens, which come multiplied by scale_log2.  Mostly scales, the scale of scores and
// the tops meet in one operation; where a top has to follow (see weigh()), or scores are huge, the products become scores first.
template <int FORMAT, int MT, int DV>
__device__ __forceinline__ void weigh_codes(Rows<MT, DV>& r, Scores<MT>& s, const float (&scale)[8], const float (&offset)[8], const float (&q_sum)[MT], float scale_log2, Weights (&w)[MT]) {
  if (!r.huge && !r.waiting) {
    float add[MT];
    bool behind = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float* x = w[mt].w;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float from = FORMAT == kInt4 ? __builtin_fmaf(offset[i], q_sum[mt], r.from[mt]) : r.from[mt];
        x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][i / 4][i % 4], scale[i], from));
      }
      add[mt] = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
      behind = behind || add[mt] > Matrix<half_t>::kLimit;
    }
    if (!__any(behind)) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) r.sum[mt] += add[mt];
      return;
    }
  }
  const float by = 1.0f / scale_log2;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float x = s[mt][i / 4][i % 4];
      s[mt][i / 4][i % 4] = (FORMAT == kInt4 ? __builtin_fmaf(x, scale[i], offset[i] * q_sum[mt]) : x * scale[i]) * by;
    }
  weigh<half_t, MT, DV>(r, s, scale_log2, w);
}

// The weights come 2^12 times as large as they are (kLift of Matrix<half_t>); scales and offsets of values are multiplied by this, so that the results are not lifted.
constexpr float kUnlift = 0x1p-12f;

// What a wavefront has of its rows: the sums of tree_attention.hpp and those of the offsets of values, which are relative to the same tops.
template <int MT, int DV>
struct QuantizedRows : Rows<MT, DV> {
  float offset[MT];
  __device__ __forceinline__ void clear_all() {
    this->clear();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) offset[mt] = 0.f;
  }
  // before: the tops when the offsets' sums were right
  __device__ __forceinline__ void follow(const float (&before)[MT], float scale_log2) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
      if (this->top[mt] != before[mt]) offset[mt] *= before[mt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((before[mt] - this->top[mt]) * scale_log2);
  }
};

// A step's share of the results: products of codes s, scales (and offsets) of keys, times scale_log2, and of values, times kUnlift, of the lane's tokens; values(v): theirs, in the
// order of value_pairs.
template <int FORMAT, typename T, int D, int MT, typename F>
__device__ __forceinline__ void add_values(const QuantizedArgs& a, QuantizedRows<MT, D / 16>& rows, Scores<MT>& s, const float (&q_sum)[MT], const float (&k_scale)[8],
                                           const float (&k_offset)[8], const float (&v_scale)[8], const float (&v_offset)[8], F values) {
  Weights w[MT];
  float before[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) before[mt] = rows.top[mt];
  weigh_codes<FORMAT, MT, D / 16>(rows, s, k_scale, k_offset, q_sum, a.scale_log2, w);
  if (FORMAT == kInt4) rows.follow(before, a.scale_log2);
  u32x4 p[MT], rest[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    if (FORMAT == kInt4)
#pragma unroll
      for (int i = 0; i < 8; ++i) rows.offset[mt] = __builtin_fmaf(w[mt].w[i], v_offset[i], rows.offset[mt]);
#pragma unroll
    for (int i = 0; i < 4; ++i) two_parts<bfloat_t>(w[mt].w[2 * i] * v_scale[2 * i], w[mt].w[2 * i + 1] * v_scale[2 * i + 1], p[mt], rest[mt], i);
  }
  u32x4 v[D / 16];
  values(v);
#pragma unroll
  for (int j = 0; j < D / 16; ++j)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      rows.o[mt][j] = Matrix<bfloat_t>::mad(v[j], p[mt], rows.o[mt][j]);
      rows.o[mt][j] = Matrix<bfloat_t>::mad(v[j], rest[mt], rows.o[mt][j]);
    }
}

// Behind the steps of codes: the nodes' steps from `step` on, every turns-th, are added as they are, their weights in two parts too.  For float16 the results are lifted meanwhile as the weights are; of bfloat16, whose values may be of any
// size, the weights' lift is taken off.
template <int FORMAT, typename T, int D, int MT>
__device__ __forceinline__ void attend_nodes(const QuantizedArgs& a, QuantizedRows<MT, D / 16>& rows, const Share& share, int old_steps, int h, int step, int turn, int turns,
                                             const u32x4 (&q)[MT][D / 32], const int (&node)[MT]) {
  constexpr int KK = D / 32, DV = D / 16;
  constexpr bool LIFT = __is_same(T, half_t);
  constexpr float kDown = LIFT ? 1.f : kUnlift;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, b = share.b, last = share.last, k_token = 8 * (n >> 2) + (n & 3);
  if (step >= last) return;
  auto times = [&](float by) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int j = 0; j < DV; ++j) rows.o[mt][j] *= by;
  };
  if (LIFT) times(1.f / kUnlift);
  const char *new_k = a.k_new.data + 2 * (b * a.k_new.batch_stride + h * a.k_new.head_stride),
             *new_v = a.v_new.data + 2 * (b * a.v_new.batch_stride + h * a.v_new.head_stride);
  bool odd = false;      // among the values is something that is no finite number
  for (; step < last; step += turns) {
    const int t0 = (step - old_steps) * kAttTile, here = a.seen_nodes - t0;
    u32x4 k[2][KK], w[MT], rest[MT];
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
    Weights weights[MT];
    weigh<half_t, MT, DV>(rows, s, a.scale_log2, weights);
    if (FORMAT == kInt4) rows.follow(before, a.scale_log2);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i) two_parts<T>(weights[mt].w[2 * i] * kDown, weights[mt].w[2 * i + 1] * kDown, w[mt], rest[mt], i);
#pragma unroll
    for (int j = 0; j < DV; ++j) {
      u32x4 t;
#pragma unroll
      for (int i = 0; i < 4; ++i) t[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        rows.o[mt][j] = Matrix<T>::mad(t, w[mt], rows.o[mt][j]);
        rows.o[mt][j] = Matrix<T>::mad(t, rest[mt], rows.o[mt][j]);
      }
    }
  }
  if (LIFT) times(kUnlift);
  if (__any(odd)) {      // a value above a weight of zero is left out; a weight above zero changes no infinity and no NaN
#pragma unroll 1
    for (int t = max(share.first - old_steps, 0) * kAttTile; t < min((last - old_steps) * kAttTile, a.seen_nodes); ++t) {
      if ((old_steps + t / kAttTile - share.first) % turns != turn) continue;
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
}

// Writes a wavefront's rows: elements [from, from + L) of the four times D / 16 that a lane has.
template <typename T, int D>
struct RowWriter {
  const QuantizedArgs& a;
  int b, h, slot, row_tile, rows_of_tile, parts;
  static constexpr int RUN = D == 96 ? D / 16 : D / 32;
  // r: of the kv head; at: of the tile
  template <int L>
  __device__ __forceinline__ void put(int r, int at, int node, int from, const float* e, float m, float s) const {
    constexpr int DV = D / 16;
    const int d = value_dim<D>(4 * ((threadIdx.x & 63) >> 4) + from / DV, from % DV);
    if (parts == 1) {
      const float by = one_over(s);
      uint32_t w[L / 2];
#pragma unroll
      for (int j = 0; j < L / 2; ++j) w[j] = pack2<T>(e[2 * j] * by, e[2 * j + 1] * by);
      store_words(a.out.data + 2 * (b * a.out.batch_stride + node * a.out.token_stride + (h * a.group + r - node * a.group) * a.out.head_stride + d), w);
    } else if (m != -INFINITY) {
      uint32_t w[L];
#pragma unroll
      for (int j = 0; j < L; ++j) w[j] = __builtin_bit_cast(uint32_t, e[j]);
      store_words(reinterpret_cast<char*>(a.part + (part_row(a, slot, h, row_tile, rows_of_tile) + at) * D + d), w);
    }
  }
  __device__ __forceinline__ void put_run(int r, int at, int node, int from, const float* e, float m, float s) const {
    if constexpr (D == 96) {
      put<4>(r, at, node, from, e, m, s);
      put<2>(r, at, node, from + 4, e + 4, m, s);
    } else {
      put<RUN>(r, at, node, from, e, m, s);
    }
  }
  __device__ __forceinline__ void put_stats(int r, int at, int node, float m, float s) const {
    if (parts != 1)
      a.stats[part_row(a, slot, h, row_tile, rows_of_tile) + at] = make_float2(m, s);
    else if (a.lse != nullptr)
      a.lse[((int64_t)b * a.nodes + node) * (a.kv_heads * a.group) + h * a.group + r - node * a.group] = log_sum<bfloat_t>(m, s, a.scale);      // (no lift is left)
  }
};

// The sums over a row's lanes, and nothing is lifted any more.
template <int FORMAT, int MT, int DV>
__device__ __forceinline__ void settle(QuantizedRows<MT, DV>& rows) {
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float s = rows.sum[mt], f = rows.offset[mt];
    s += __shfl_xor(s, 16);
    rows.sum[mt] = (s + __shfl_xor(s, 32)) * kUnlift;
    if (FORMAT == kInt4) {
      f += __shfl_xor(f, 16);
      rows.offset[mt] = f + __shfl_xor(f, 32);
    }
  }
}

// The rows of a wavefront that has a head (and a part of its tokens) to itself.
template <typename T, int D, int MT>
__device__ __forceinline__ void write_rows(const RowWriter<T, D>& to, const QuantizedRows<MT, D / 16>& rows, int first_row, int first_at, const int (&node)[MT]) {
  constexpr int DV = D / 16, RUN = RowWriter<T, D>::RUN;
  const int lane = threadIdx.x & 63, n = lane & 15;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = first_row + mt * 16 + n, at = first_at + mt * 16 + n;
    if (r >= to.a.rows) continue;
#pragma unroll
    for (int from = 0; from < 4 * DV; from += RUN) {
      float e[RUN];
#pragma unroll
      for (int j = 0; j < RUN; ++j) e[j] = rows.o[mt][(from + j) % DV][(from + j) / DV] + rows.offset[mt];
      to.put_run(r, at, node[mt], from, e, rows.top[mt], rows.sum[mt]);
    }
    if (lane < 16) to.put_stats(r, at, node[mt], rows.top[mt], rows.sum[mt]);
  }
}

// The parts of a row meet: a workgroup to a row, since a lone long sequence has hundreds of parts.  Groups of D / 4 threads take parts in turns, four elements to a thread, and meet
// in LDS.  (A part that its rows saw nothing of has no top and has not been written; it may have a NaN for a sum, which is what the row is then.)
template <typename T, int D, int THREADS>
__global__ void __launch_bounds__(THREADS) quantized_join_kernel(const QuantizedArgs a, int rows_of_tile, Divide by_rows, Divide by_heads, Divide by_tile) {
  constexpr int W = D / 4, G = THREADS / W, WAVES = THREADS / 64;
  __shared__ float factors[THREADS], wave_tops[WAVES], wave_sums[WAVES];
  __shared__ f32x4 meet[G][W];
  const uint32_t bh = by_rows.of(blockIdx.x), r = blockIdx.x - bh * a.rows, b = by_heads.of(bh), h = bh - b * a.kv_heads, row_tile = by_tile.of(r);
  const int2 place = a.places[b];
  const int parts = place.y;
  if (parts == 1) return;      // its workgroup has written the result
  const int64_t first = part_row(a, place.x, h, row_tile, rows_of_tile) + (r - row_tile * rows_of_tile), step = (int64_t)a.kv_heads * a.row_tiles * rows_of_tile;
  const int wave = threadIdx.x >> 6, group = threadIdx.x / W, at = 4 * (threadIdx.x % W);
  float m = -INFINITY, s = 0.f;
  f32x4 e{0, 0, 0, 0};
  for (int p0 = 0; p0 < parts; p0 += THREADS) {
    const int p = p0 + (int)threadIdx.x, here = min(THREADS, parts - p0);
    const float2 mine = p < parts ? a.stats[first + p * step] : make_float2(-INFINITY, 0.f);
    const float top = wave_all(mine.x, [](float x, float y) { return fmaxf(x, y); });
    if ((threadIdx.x & 63) == 0) wave_tops[wave] = top;
    __syncthreads();
    float next = m;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) next = fmaxf(next, wave_tops[w]);
    const float less = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - next) * a.scale_log2);
    const float f = mine.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mine.x - next) * a.scale_log2);
    const float add = wave_all(f * mine.y, [](float x, float y) { return x + y; });
    factors[threadIdx.x] = f;
    if ((threadIdx.x & 63) == 0) wave_sums[wave] = add;
    __syncthreads();
    s *= less;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += wave_sums[w];
    e *= less;
    m = next;
    if (group < G)
#pragma unroll 4
      for (int i = group; i < here; i += G) {
        const float by = factors[i];
        const f32x4 v = *reinterpret_cast<const f32x4*>(a.part + (first + (p0 + i) * step) * D + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] += by == 0.f ? 0.f : by * v[j];
      }
    __syncthreads();
  }
  if (group < G) meet[group][threadIdx.x % W] = e;
  __syncthreads();
  const int node = a.by_group.of(r), head = h * a.group + r - node * a.group;
  if (group == 0) {
#pragma unroll
    for (int i = 1; i < G; ++i) e += meet[i][threadIdx.x];
    const float by = one_over(s);
    *reinterpret_cast<uint2*>(a.out.data + 2 * (b * a.out.batch_stride + node * a.out.token_stride + head * a.out.head_stride + at)) =
        make_uint2(pack2<T>(e[0] * by, e[1] * by), pack2<T>(e[2] * by, e[3] * by));
  }
  if (a.lse != nullptr && threadIdx.x == 0) a.lse[((int64_t)b * a.nodes + node) * (a.kv_heads * a.group) + head] = log_sum<bfloat_t>(m, s, a.scale);
}

// The kernel for few rows: as tree_attention_kernel, with steps of codes in front of those of the nodes.  A lane reads a quarter of each of two keys (16 to 64
// bytes in a row) and its dimensions of eight values; the next step's are on their way while this one's are used, as a step of codes has half or a quarter of the bytes
// in flight that one of numbers has.
template <int FORMAT, typename T, int D, int MT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, D <= 128 ? 2 : 1) quantized_attention_kernel(const QuantizedArgs a) {
  typedef Held<FORMAT, D> H;
  constexpr int KK = D / 32, DV = D / 16, R = 16 * MT;
  constexpr int RUN = RowWriter<T, D>::RUN;      // a wavefront adds up so many of a lane's 4 DV results at a time in the end
  // the tokens of a step of each wavefront, and in the end the wavefronts' results
  constexpr int kTokens = 2 * kAttTile * H::ROW, kSums = 4 * DV * MT * 64 * (int)sizeof(float);
  __shared__ __align__(16) char tokens[WAVES][kTokens > kSums ? kTokens : kSums];
  __shared__ float offsets[WAVES][MT][16];
  __shared__ float2 tops[WAVES][MT][16];
  __shared__ __align__(16) int64_t places[WAVES][kAttTile];
  __shared__ __align__(16) float scales_of[WAVES][FORMAT == kInt4 ? 4 : 2][kAttTile];      // of keys, of values, offsets of keys, of values
  const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  int slot, first_head, row_tile;
  place_group(a, a.heads_at_once, slot, first_head, row_tile);
  const int turns = a.turns, turn = wave / a.heads_at_once, mate = wave - turn * a.heads_at_once, h = first_head + mate;
  const Share share = share_of(a, slot);
  if (share.b < 0) return;
  const int b = share.b, old_steps = steps_of(share.len), last = share.last, last_old = min(last, old_steps);
  if (share.part == 0 && first_head == 0 && row_tile == 0 && threadIdx.x == 0 && a.places != nullptr) a.places[b] = make_int2(slot, share.parts);

  u32x4 q[MT][KK];
  float q_sum[MT] = {};
  int node[MT];
  int step = share.first + turn;
  Lookup next = ask_held(a, share, last_old, step);
  load_quarters<FORMAT, D, MT>(a, b, h, row_tile * R, q, node);
  if (FORMAT == kInt4) sum_queries<T, D, MT>(q, q_sum);
  QuantizedRows<MT, DV> rows;
  rows.clear_all();
  const char *cache_k = a.cache.k + h * a.cache.head_stride, *cache_v = a.cache.v + h * a.cache.head_stride;
  const uint32_t* scales = (lane < kAttTile ? a.k_scales : a.v_scales) + h * a.scale_head;
  // A wavefront loads the keys and values of a step as they lie, 16 bytes to a lane and neighbours to neighbours, and turns them round in LDS: a lane's own quarter of a key is
  // next to no other lane's, and the cache would be asked for every lane by itself (four times the accesses, 500 a step, which is what bound it).
  struct Tokens {
    u32x4 k[H::LOADS], v[H::LOADS];
    uint32_t word, there;
  };
  char* const turn_k = tokens[wave];
  char* const turn_v = tokens[wave] + kAttTile * H::ROW;
  auto load = [&](int step, Tokens& x) {
    const HeldPlace mine = held_place(a, share, last_old, step, next);
    // loads come back in their order: the places of the step behind this one are asked for in front of its tokens, so that nobody waits for those to look a place up
    next = ask_held(a, share, last_old, step + turns);
    x.word = scales[mine.scale_at];
    if (!mine.there) x.word = lane >= kAttTile ? 0u : FORMAT == kInt4 ? 0x3f80u : 0x3f800000u;      // values of 0, keys (which have no score) of scale 1
    if (lane < kAttTile) places[wave][lane] = mine.at;
    x.there = (uint32_t)__ballot(mine.there);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < H::LOADS; ++i) {
      const int piece = 64 * i + lane, row = min(piece / H::PIECES, kAttTile - 1);
      const int key = 8 * ((row & 15) >> 2) + (row & 3) + 4 * (row >> 4);      // as score() numbers the tokens
      x.k[i] = load_piece<H::BYTES % 128 == 0>(cache_k + places[wave][key] + 16 * (piece % H::PIECES));
      x.v[i] = load_piece<H::BYTES % 128 == 0>(cache_v + places[wave][row] + 16 * (piece % H::PIECES));
    }
  };
  auto attend = [&](Tokens& x) {
    const bool all = x.there == 0xffffffffu;
    const float by = lane >= kAttTile ? kUnlift : a.scale_log2;
    scales_of[wave][lane >> 5][lane & 31] = scale_of<FORMAT>(x.word) * by;
    if (FORMAT == kInt4) scales_of[wave][2 + (lane >> 5)][lane & 31] = offset_of(x.word) * by;
#pragma unroll
    for (int i = 0; i < H::LOADS; ++i) {
      const int piece = 64 * i + lane, at = piece / H::PIECES * H::ROW + 16 * (piece % H::PIECES);
      if (32 * H::PIECES % 64 != 0 && piece >= 32 * H::PIECES) continue;
      *reinterpret_cast<u32x4*>(turn_k + at) = x.k[i];
      *reinterpret_cast<u32x4*>(turn_v + at) = x.v[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    auto eight = [&](int which, float (&to)[8]) {      // of the lane's tokens
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x4 p = *reinterpret_cast<const f32x4*>(&scales_of[wave][which][8 * g + 4 * i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) to[4 * i + j] = p[j];
      }
    };
    float k_scale[8], v_scale[8], k_offset[8], v_offset[8];
    eight(0, k_scale);
    eight(1, v_scale);
    if (FORMAT == kInt4) {
      eight(2, k_offset);
      eight(3, v_offset);
    }
    u32x4 k[2][KK];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const Codes<H::KW> codes = load_codes<H::KW>(turn_k + (16 * half + n) * H::ROW + g * (H::BYTES / 4));
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) k[half][kk] = key_operand<FORMAT, T>(codes, kk);
    }
    Codes<H::VW> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = load_value<FORMAT, D>(turn_v + (8 * g + i) * H::ROW, n);
    Scores<MT> s;
    score<T, D, MT>(q, k, s);
    if (!all) {
      uint32_t seen[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) seen[mt] = (x.there >> (8 * g)) & 0xffu;
      mask<MT>(s, seen);
      // a token that is not there was read from a place that is, and counts as zeros
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < H::VW; ++j) v[i].w[j] = (x.there >> (8 * g + i)) & 1 ? v[i].w[j] : 0u;
    }
    add_values<FORMAT, T, D, MT>(a, rows, s, q_sum, k_scale, k_offset, v_scale, v_offset, [&](u32x4(&to)[DV]) {
      uint32_t pairs[4][DV];
#pragma unroll
      for (int i = 0; i < 4; ++i) value_pairs<FORMAT, DV>(v[2 * i], v[2 * i + 1], pairs[i]);
#pragma unroll
      for (int j = 0; j < DV; ++j) to[j] = u32x4{pairs[0][j], pairs[1][j], pairs[2][j], pairs[3][j]};
    });
  };
  if (step < last_old) {
    Tokens x, y;
    if constexpr (MT == 1 || H::LOADS <= 2) {      // (for two tiles of rows and 8 bits there are no registers for a step ahead)
      load(step, x);
#pragma unroll 1
      for (; step < last_old; step += turns) {
        load(step + turns, y);
        attend(x);
        x = y;
      }
    } else {
#pragma unroll 1
      for (; step < last_old; step += turns) {
        load(step, x);
        attend(x);
      }
    }
  }

  attend_nodes<FORMAT, T, D, MT>(a, rows, share, old_steps, h, step, turn, turns, q, node);
  settle<FORMAT, MT, DV>(rows);
  const RowWriter<T, D> to{a, b, h, slot, row_tile, R, share.parts};
  if (turns == 1) {      // every wavefront has a head to itself
    write_rows<T, D, MT>(to, rows, row_tile * R, 0, node);
    return;
  }
  // the rows of the wavefronts of a head meet: each adds up its part of the elements
  auto sums_of = [&](int w) { return reinterpret_cast<float*>(tokens[w]); };
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    if (g == 0) {
      tops[wave][mt][n] = make_float2(rows.top[mt], rows.sum[mt]);
      offsets[wave][mt][n] = rows.offset[mt];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < DV; ++j) sums_of(wave)[((mt * 4 + i) * DV + j) * 64 + lane] = rows.o[mt][j][i];
  }
  __syncthreads();
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = row_tile * R + mt * 16 + n;
    float m = -INFINITY, s = 0.f, plus = 0.f, f[WAVES];
#pragma unroll
    for (int t = 0; t < WAVES; ++t)
      if (t < turns) m = fmaxf(m, tops[mate + t * a.heads_at_once][mt][n].x);
#pragma unroll
    for (int t = 0; t < WAVES; ++t) {
      f[t] = 0.f;
      if (t >= turns) continue;
      const float2 x = tops[mate + t * a.heads_at_once][mt][n];
      f[t] = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x.x - m) * a.scale_log2);
      s += x.y * f[t];
      if (FORMAT == kInt4) plus += offsets[mate + t * a.heads_at_once][mt][n] * f[t];
    }
    if (r >= a.rows) continue;
    for (int from = turn * RUN; from < 4 * DV; from += turns * RUN) {
      float e[RUN];
#pragma unroll
      for (int j = 0; j < RUN; ++j) {
        e[j] = plus;
#pragma unroll
        for (int t = 0; t < WAVES; ++t)
          if (t < turns) e[j] += sums_of(mate + t * a.heads_at_once)[(mt * 4 * DV + from + j) * 64 + lane] * f[t];
      }
      to.put_run(r, mt * 16 + n, node[mt], from, e, m, s);
    }
    if (g == 0 && turn == 0) to.put_stats(r, mt * 16 + n, node[mt], m, s);
  }
}

// The kernel for many rows: WAVES wavefronts with 16 * MT rows each take every step of codes together.  They are loaded once for all of them, a step ahead, and come into LDS as the numbers that the products
// want, two steps in turns, so that they are taken apart once and not by every wavefront:
//   K: pieces of 8 elements [D / 8][32 tokens] as in tree_attention_wide_kernel, the elements in the order of key_operand;
//   V: turned, [4 groups of 8 tokens][D] of 16 bytes, element d of sixteen in place (d + d / 16) % 16 of them, so that neither four neighbours of a piece nor the lanes that read D / 16
//      elements apart meet in a bank;
//   scales (and offsets): of the keys times scale_log2, of the values times kUnlift.
// A unit of work is 16 bytes of a token's key, or 4 bytes of each of four tokens' values.
template <int FORMAT, typename T, int D, int MT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, D <= 128 ? 2 : 1) quantized_attention_wide_kernel(const QuantizedArgs a) {
  typedef Held<FORMAT, D> H;
  constexpr int KK = D / 32, DV = D / 16, R = 16 * MT * WAVES, THREADS = WAVES * 64;
  constexpr int K_UNITS = 32 * H::PIECES, V_WORDS = H::BYTES / 4, V_UNITS = 8 * V_WORDS, U = (K_UNITS + V_UNITS + THREADS - 1) / THREADS;
  constexpr int EACH = 32 / H::BITS, SETS = FORMAT == kInt4 ? 4 : 2;      // codes of a word
  __shared__ __align__(16) char lds_k[2][4 * D * 16], lds_v[2][4 * D * 16];
  __shared__ __align__(16) float lds_scales[2][SETS][kAttTile];
  __shared__ __align__(16) int64_t places[2 * WAVES][kAttTile];      // [step][token]
  __shared__ uint32_t lds_words[2 * WAVES][2][kAttTile], lds_there[2 * WAVES];
  const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  int slot, h, row_tile;
  place_group(a, 1, slot, h, row_tile);
  const Share share = share_of(a, slot);
  if (share.b < 0) return;
  const int b = share.b, old_steps = steps_of(share.len), first = share.first, last_old = min(share.last, old_steps);
  if (share.part == 0 && h == 0 && row_tile == 0 && threadIdx.x == 0 && a.places != nullptr) a.places[b] = make_int2(slot, share.parts);

  // Places and scales are looked up for as many steps at a time as there are wavefronts, one by each, that many steps before they are needed.  Loads are up to three steps ahead.
  static_assert(WAVES >= 4, "places of the steps that loads are ahead by");
  const uint32_t* scales = (lane < kAttTile ? a.k_scales : a.v_scales) + h * a.scale_head;
  struct Found {
    HeldPlace place;
    uint32_t word;
  };
  auto find = [&](int step, const Lookup& l) {
    Found f{held_place(a, share, last_old, step, l), 0u};
    f.word = scales[f.place.scale_at];
    if (!f.place.there) f.word = lane >= kAttTile ? 0u : FORMAT == kInt4 ? 0x3f80u : 0x3f800000u;
    return f;
  };
  auto keep_places = [&](int step, const Found& f) {
    const int at = (step - first) & (2 * WAVES - 1);
    if (lane < kAttTile) places[at][lane] = f.place.at;
    lds_words[at][lane >> 5][lane & 31] = f.word;
    const uint32_t there = (uint32_t)__ballot(f.place.there);
    if (lane == 0) lds_there[at] = there;
  };
  keep_places(first + wave, find(first + wave, ask_held(a, share, last_old, first + wave)));
  u32x4 q[MT][KK];
  float q_sum[MT] = {};
  int node[MT];
  load_quarters<FORMAT, D, MT>(a, b, h, row_tile * R + wave * 16 * MT, q, node);
  if (FORMAT == kInt4) sum_queries<T, D, MT>(q, q_sum);
  const bool works = row_tile * R + wave * 16 * MT < a.rows;      // a wavefront without rows only loads
  QuantizedRows<MT, DV> rows;
  rows.clear_all();
  const char *cache_k = a.cache.k + h * a.cache.head_stride, *cache_v = a.cache.v + h * a.cache.head_stride;
  auto load = [&](int step, u32x4 (&x)[U]) {
    const int64_t* at = places[(step - first) & (2 * WAVES - 1)];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = (int)threadIdx.x + i * THREADS;
      if (u < K_UNITS) {
        x[i] = *reinterpret_cast<const u32x4*>(cache_k + at[u / H::PIECES] + 16 * (u % H::PIECES));
      } else {
        const int v = min(u - K_UNITS, V_UNITS - 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = *reinterpret_cast<const uint32_t*>(cache_v + at[4 * (v / V_WORDS) + j] + 4 * (v % V_WORDS));
      }
    }
  };
  auto keep = [&](int step, const u32x4 (&x)[U]) {
    const int at = (step - first) & (2 * WAVES - 1);
    const uint32_t there = (uint32_t)scalar((int)lds_there[at]);
    if (threadIdx.x < 64) {
      const uint32_t word = lds_words[at][lane >> 5][lane & 31];
      const float by = lane >= kAttTile ? kUnlift : a.scale_log2;
      lds_scales[step & 1][lane >> 5][lane & 31] = scale_of<FORMAT>(word) * by;
      if (FORMAT == kInt4) lds_scales[step & 1][2 + (lane >> 5)][lane & 31] = offset_of(word) * by;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = (int)threadIdx.x + i * THREADS;
      if (u < K_UNITS) {
        const int token = u / H::PIECES, place = ((token >> 2) & 1) * 16 + 4 * (token >> 3) + (token & 3);      // as score() numbers the tokens
        constexpr int P = FORMAT == kInt4 ? 4 : 2;
        const Codes<4> codes{{x[i][0], x[i][1], x[i][2], x[i][3]}};
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const int piece = u % H::PIECES * P + p;
          *reinterpret_cast<u32x4*>(lds_k[step & 1] + (piece * kAttTile + (place ^ (piece & 15))) * 16) = key_operand<FORMAT, T>(codes, p);
        }
      } else if ((K_UNITS + V_UNITS) % THREADS == 0 || u < K_UNITS + V_UNITS) {
        const int v = u - K_UNITS, four = v / V_WORDS, d0 = EACH * (v % V_WORDS);
        Codes<1> c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j].w[0] = (there >> (4 * four + j)) & 1 ? x[i][j] : 0u;      // (a token that is not there was read from a place that is)
        uint32_t low[EACH], high[EACH];
        value_pairs<FORMAT, EACH>(c[0], c[1], low);
        value_pairs<FORMAT, EACH>(c[2], c[3], high);
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
          const int d = d0 + e;
          *reinterpret_cast<uint2*>(lds_v[step & 1] + ((four >> 1) * D + (d & ~15) + ((d + (d >> 4)) & 15)) * 16 + (four & 1) * 8) = make_uint2(low[e], high[e]);
        }
      }
    }
  };
  auto attend = [&](int step) {
    u32x4 k[2][KK];
    Scores<MT> s;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const int piece = g * KK + kk;
        k[half][kk] = *reinterpret_cast<const u32x4*>(lds_k[step & 1] + (piece * kAttTile + half * 16 + (n ^ (piece & 15))) * 16);
      }
    score<T, D, MT>(q, k, s);
    float k_scale[8], v_scale[8], k_offset[8], v_offset[8];
    auto eight = [&](int which, float (&to)[8]) {      // of the lane's tokens
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x4 p = *reinterpret_cast<const f32x4*>(&lds_scales[step & 1][which][8 * g + 4 * i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) to[4 * i + j] = p[j];
      }
    };
    eight(0, k_scale);
    eight(1, v_scale);
    if (FORMAT == kInt4) {
      eight(2, k_offset);
      eight(3, v_offset);
    }
    const uint32_t there = (uint32_t)scalar((int)lds_there[(step - first) & (2 * WAVES - 1)]);
    if (there != 0xffffffffu) {
      uint32_t seen[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) seen[mt] = (there >> (8 * g)) & 0xffu;
      mask<MT>(s, seen);
    }
    add_values<FORMAT, T, D, MT>(a, rows, s, q_sum, k_scale, k_offset, v_scale, v_offset, [&](u32x4(&v)[DV]) {
#pragma unroll
      for (int j = 0; j < DV; ++j) {
        const int d = value_dim<D>(n, j);
        v[j] = *reinterpret_cast<const u32x4*>(lds_v[step & 1] + (g * D + (d & ~15) + ((d + (d >> 4)) & 15)) * 16);
      }
    });
  };

  if (first < last_old) {
    __syncthreads();
    u32x4 x[U], y[U];
    load(first, x);
    constexpr bool TWO = FORMAT != kInt4 || D < 128;      // two steps of loads are on their way, if there are registers for them (100 rows in 8 bits 154 us, with one 162)
    if (TWO) load(first + 1, y);
    keep(first, x);
    __syncthreads();
#pragma unroll 1
    for (int step = first; step < last_old; step += TWO ? 2 : 1) {
      const bool ahead = ((step - first) & (WAVES - 1)) == 0;
      Lookup after{};
      if (ahead) after = ask_held(a, share, last_old, step + WAVES + wave);
      load(TWO ? step + 2 : step + 1, x);
      Found found{};
      if (ahead) found = find(step + WAVES + wave, after);
      if (works) attend(step);
      keep(step + 1, TWO ? y : x);
      if (ahead) keep_places(step + WAVES + wave, found);
      __syncthreads();
      if constexpr (TWO) {
        if (step + 1 >= last_old) break;
        load(step + 3, y);
        if (works) attend(step + 1);
        keep(step + 2, x);
        __syncthreads();
      }
    }
  }
  if (!works) return;
  attend_nodes<FORMAT, T, D, MT>(a, rows, share, old_steps, h, max(first, old_steps), 0, 1, q, node);
  settle<FORMAT, MT, DV>(rows);
  write_rows<T, D, MT>(RowWriter<T, D>{a, b, h, slot, row_tile, R, share.parts}, rows, row_tile * R + wave * 16 * MT, wave * 16 * MT, node);
}

}  // namespace dpllm
