// Keys and values held in 8 or 4 bits: a head of a token is its codes and one 32-bit word.
//   e4m3  the smallest scale 2^k with which the largest value is at most 448; codes are x / scale, rounded (a division that rounds nothing)
//   int8  scale = max |x| / 127, codes 127 x / max |x| rounded to whole numbers
//   int4  offset = (lo + hi) / 2 in bfloat16, scale = an eighth of the larger distance from it, upwards to bfloat16; n = floor((x - offset) / scale) of
//         -8 ... 7 stands for offset + scale (n + 1/2): 16 levels, none of them wasted on a second zero, and no error above half a scale.  Kept as sign and magnitude (n or
//         -1 - n), the codes of 2i and 2i + 1 in byte i, which are the low bits of an e4m3 number once shifted: that type counts in even steps up to 15.
// A largest value (or distance) below 2^-100 counts as that.  A head with a value that is no finite number has a NaN for a scale.
#pragma once
#include "lanes.hpp"
#include "token_common.hpp"

namespace dpllm {

constexpr int kE4m3 = DPLLM_CACHE_E4M3, kInt8 = DPLLM_CACHE_INT8, kInt4 = DPLLM_CACHE_INT4;
constexpr uint32_t kNan32 = 0x7fc00000u;
constexpr float kLeast = 0x1p-100f;

// One layer of such a cache.  Strides of codes in bytes, of scales in words; tokens are found as in a cache of numbers.
struct QuantizedView {
  char *k, *v;
  uint32_t *k_scales, *v_scales;
  int64_t layer, page_stride, token, head, scale_layer, scale_page, scale_token, scale_head;
  const int32_t* table;
  int64_t table_stride;
  Divide by_page;
  int pages, page, pages_per_seq;
  // Where token t of sequence b starts; false: no page holds it.
  __device__ __forceinline__ bool find(int b, uint32_t t, int64_t* at, int64_t* scale_at) const {
    const uint32_t j = by_page.of(t), in_page = t - j * (uint32_t)page;
    if (j >= (uint32_t)pages_per_seq) return false;
    const int id = table == nullptr ? b : table[b * table_stride + j];
    if ((uint32_t)id >= (uint32_t)pages) return false;
    *at = (int64_t)id * page_stride + (int64_t)in_page * token;
    *scale_at = (int64_t)id * scale_page + (int64_t)in_page * scale_token;
    return true;
  }
};

// ---- codes to numbers ----
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// The four levels in the lower (ODD: upper) halves of four bytes, a sign and a magnitude m each, as e4m3 numbers of size (2m + 1) / 512: that type's numbers below 1/32 are whole 512ths, so the
// size's byte is 2m + 1, which comes out of a table of eight.
template <bool ODD>
__device__ __forceinline__ uint32_t level_bytes(uint32_t x) {
  const uint32_t size = __builtin_amdgcn_perm(0x0f0d0b09u, 0x07050301u, (ODD ? x >> 4 : x) & 0x07070707u);
  return ((ODD ? x : x << 4) & 0x80808080u) | (size & ~0x80808080u);
}

// Two of four codes (the lower two or the upper two bytes; of int4 level_bytes) as T.
template <int FORMAT, typename T>
__device__ __forceinline__ uint32_t two_codes(uint32_t w, bool upper) {
  constexpr float kBy = FORMAT == kInt4 ? 256.f : 1.f;
  if constexpr (FORMAT == kInt8 && sizeof(T) == 2 && __is_same(T, half_t)) {
    // 1024 + (code + 128) in the lower bits of a half, of which 1152 are taken off
    const uint32_t p = __builtin_amdgcn_perm(0x64646464u, w ^ 0x80808080u, upper ? 0x04030402u : 0x04010400u);
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, p) - f16x2{(half_t)1152.f, (half_t)1152.f});
  } else if constexpr (FORMAT == kInt8) {
    const int s = upper ? 16 : 0;
    const float a = (float)(int8_t)(w >> s), b = (float)(int8_t)(w >> (s + 8));
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);      // a whole number below 256 is its upper half
  } else if constexpr (__is_same(T, half_t)) {
    return __builtin_bit_cast(uint32_t, upper ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, kBy, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, kBy, false));
  } else {
    return __builtin_bit_cast(uint32_t, upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, kBy, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, kBy, false));
  }
}

// The numbers of a head's word.
template <int FORMAT>
__device__ __forceinline__ float scale_of(uint32_t w) {
  return __uint_as_float(FORMAT == kInt4 ? w << 16 : w);
}
__device__ __forceinline__ float offset_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }      // int4 only

// What four codes (of int4 level_bytes) stand for.
template <int FORMAT>
__device__ __forceinline__ void four_values(uint32_t w, uint32_t scales, float (&x)[4]) {
  const float s = scale_of<FORMAT>(scales);
  if constexpr (FORMAT == kInt8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i)) * s;
  } else {
    constexpr float kBy = FORMAT == kInt4 ? 256.f : 1.f;
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, kBy, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, kBy, true);
    const float c[4] = {a[0], a[1], b[0], b[1]};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = FORMAT == kInt4 ? __builtin_fmaf(c[i], s, offset_of(scales)) : c[i] * s;
  }
}

// ---- numbers to codes ----
// What a head's word takes: the largest size, of int4 the lowest and highest value; infinite where a value is no finite number.
struct Extent {
  float most, lo, hi;
};
// (of values that may be signaling NaN, which the compiler would see to first)
__device__ __forceinline__ float least_of(float a, float b, float c) {
  float r;
  asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float most_of(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float most_size(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
template <int FORMAT, int E>
__device__ __forceinline__ void extend(Extent& e, const float (&x)[E]) {
  bool nan = false;
#pragma unroll
  for (int i = 0; i < E; i += 2) {
    nan = nan || __builtin_isunordered(x[i], x[i + 1]);
    if (FORMAT == kInt4) {
      e.lo = least_of(e.lo, x[i], x[i + 1]);
      e.hi = most_of(e.hi, x[i], x[i + 1]);
    } else {
      e.most = most_size(e.most, x[i], x[i + 1]);
    }
  }
  if (nan) e.most = e.hi = INFINITY;
}
struct Coder {
  uint32_t word;
  float scale, offset, by, top;      // by: 1 / scale, or 127 / top, to 2^-22
  bool bad;
};
template <int FORMAT>
__device__ __forceinline__ Coder coder_of(const Extent& e) {
#pragma clang fp contract(off)
  Coder c{};
  if (FORMAT == kInt4) {
    const float middle = e.lo * 0.5f + e.hi * 0.5f;
    c.offset = (float)(bfloat_t)middle;
    const float reach = fmaxf(e.hi - c.offset, c.offset - e.lo);
    const uint32_t up = (__float_as_uint(fmaxf(reach, kLeast) * 0.125f) + 0xffffu) & 0xffff0000u;
    c.scale = __uint_as_float(up);
    c.by = __builtin_amdgcn_rcpf(c.scale);
    c.bad = up >= 0x7f800000u || !__builtin_isfinite(c.offset);
    c.word = c.bad ? kNan32 >> 16 : (reach > 0.f ? up >> 16 : 0u) | __float_as_uint(c.offset);      // (0: all values are the offset)
  } else {
    c.bad = e.most == INFINITY;
    c.top = fmaxf(e.most, kLeast);
    if (FORMAT == kInt8) {
      // the quotient to the last bit: its remainder is known exactly
      constexpr float k127th = 1.f / 127.f;
      const float near = c.top * k127th;
      c.scale = __builtin_fmaf(__builtin_fmaf(-127.f, near, c.top), k127th, near);
      c.by = __builtin_amdgcn_rcpf(c.scale);      // (that of the largest float is none that it gives)
    } else {
      // top = m 2^e, 448 = 1.75 2^8: the exponent is e - 8, one more if m is above 1.75
      const uint32_t bits = __float_as_uint(c.top), exponent = (bits >> 23) - 8u + ((bits & 0x7fffffu) > 0x600000u ? 1u : 0u);
      c.scale = __uint_as_float(exponent << 23);
      c.by = __uint_as_float((254u - exponent) << 23);
    }
    c.word = c.bad ? kNan32 : __float_as_uint(c.scale);
  }
  return c;
}

// Values as codes, side by side.  The quotients of int8 and int4 are products with the reciprocal; where it matters remainders decide, which are exact for values of 16 bits (x 127 and n top have 18 bits,
// n scale has 12).
template <int FORMAT, int E>
__device__ __forceinline__ void codes_of(const Coder& c, const float (&x)[E], uint32_t (&w)[FORMAT == kInt4 ? (E + 7) / 8 : E / 4]) {
#pragma clang fp contract(off)
  if constexpr (FORMAT == kE4m3) {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * c.by, x[4 * i + 1] * c.by, 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * c.by, x[4 * i + 3] * c.by, (int)w[i], true);
    }
  } else if constexpr (FORMAT == kInt8) {
    float n[E], off = 0.f;
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const float t = x[i] * c.by, u = x[i + 1] * c.by;
      n[i] = __builtin_rintf(t);
      n[i + 1] = __builtin_rintf(u);
      off = most_size(off, t - n[i], u - n[i + 1]);
    }
    if (__any(off > 0.5f - 0x1p-14f)) {
      asm volatile("");      // (a branch: few wavefronts have such a value, and all would take the remainders)
      const float down = c.top > 0x1p100f ? 0x1p-20f : 1.f, top = c.top * down;      // 127 x stays a float
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float rest = __builtin_fmaf(-n[i], top, x[i] * down * 127.f), twice = 2.f * __builtin_fabsf(rest);
        const bool odd = ((int)n[i] & 1) != 0;
        if (twice > top || (twice == top && odd)) n[i] += __builtin_copysignf(1.f, rest);
      }
    }
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      w[i] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i] |= ((uint32_t)(int)n[4 * i + j] & 0xffu) << (8 * j);
    }
  } else {
    // The magnitude, n or -1 - n, is the whole part of |x - offset| / scale, which a product that is a little large gives or exceeds by 1: so the remainder's sign decides.  Values on a border, where the remainder
    // is 0, belong to the level above, which for negative ones is the smaller magnitude; they are as many as five in a thousand of bfloat16 values, so all go this way.  -0.0 less an offset of 0 is -0.0,
    // which has no smaller magnitude and is not below the offset: 0 is added, which makes it 0 and leaves all other differences as they are.
    const float by = c.by * (1.f + 0x1p-20f);
#pragma unroll
    for (int i = 0; i < (E + 7) / 8; ++i) {
      w[i] = 0;
#pragma unroll
      for (int j = 0; j < (E < 8 ? E : 8); ++j) {
        const float d = (x[8 * i + j] - c.offset) + 0.f, whole = __builtin_truncf(fminf(__builtin_fabsf(d) * by, 7.5f)), rest = __builtin_fmaf(-whole, c.scale, __builtin_fabsf(d));
        const uint32_t negative = __float_as_uint(d) >> 31;
        const uint32_t m = (uint32_t)((int)whole + ((__builtin_bit_cast(int, rest) - (int)negative) >> 31));
        w[i] |= (m | negative << 3) << (4 * j);
      }
    }
  }
  if (c.bad)
#pragma unroll
    for (uint32_t& v : w) v = 0;
}
// Four nibbles side by side to the lower halves of four bytes.
__device__ __forceinline__ uint32_t apart(uint32_t w) {
  w = (w & 0xffu) | ((w & 0xff00u) << 8);
  return (w & 0x000f000fu) | ((w & 0x00f000f0u) << 4);
}

// ---- append ----
constexpr int kQuantThreads = 256;
constexpr int kQuantTokens = 64;      // most tokens to a workgroup

struct QuantizeArgs {
  QuantizedView cache;           // the first layer written
  Heads k, v;                    // [layers][batch][tokens][heads][head_dim]
  int64_t k_layer, v_layer;
  const int32_t *lens, *path, *count;
  int64_t path_stride;
  Divide by_heads;
  int tokens, heads, head_dim, units, lanes, log_lanes, at_a_time;      // units of E elements to a head, lanes that share one
};

// A group of `lanes` lanes (a power of two) quantises a head of a token: its values are read once into registers where there are no more units than lanes (ONE), the next head's while this one is
// quantised, else twice.
// Grid: (at_a_time tokens, 2 layers + (keys, values), sequence), whose places are looked up first.  A unit is N pieces of 16 bytes, two where a head divides into those (what is done once for a head and lane
// is as much as for 16 elements); N = 0: four elements that are read and written by themselves, of which the last unit may have fewer.
// Bound by the latency of a launch for single tokens, by memory and the vector unit for prompts.
template <int FORMAT, typename T, int N, bool ONE>
__global__ void __launch_bounds__(kQuantThreads) quantized_append_kernel(const QuantizeArgs a) {
  constexpr bool WIDE = N > 0;
  constexpr int P = Piece<T>::E, E = WIDE ? N * P : 4, W = FORMAT == kInt4 ? (E + 7) / 8 : E / 4;
  typedef typename Piece<T>::type piece;
  __shared__ int64_t places[kQuantTokens][2];
  __shared__ int nodes[kQuantTokens];      // -1: none goes there
  const int b = blockIdx.z, layer = blockIdx.y >> 1, first = blockIdx.x * a.at_a_time;
  const bool values = blockIdx.y & 1;
  int n = a.count == nullptr ? a.tokens : min(a.count[b], a.tokens);
  n = min(n - first, a.at_a_time);
  if (n <= 0) return;
  const int base = a.lens[b];
  if (base < 0) return;
  if ((int)threadIdx.x < n) {
    const uint32_t place = first + threadIdx.x;
    int node = a.path == nullptr ? (int)place : a.path[b * a.path_stride + place];
    int64_t at = 0, scale_at = 0;
    if ((uint32_t)node >= (uint32_t)a.tokens || (uint32_t)base + place > 0x7fffffffu || !a.cache.find(b, (uint32_t)base + place, &at, &scale_at)) node = -1;
    nodes[threadIdx.x] = node;
    places[threadIdx.x][0] = at;
    places[threadIdx.x][1] = scale_at;
  }
  __syncthreads();
  const Heads& from = values ? a.v : a.k;
  const T* src = reinterpret_cast<const T*>(from.data) + layer * (values ? a.v_layer : a.k_layer) + b * from.batch_stride;
  char* codes = (values ? a.cache.v : a.cache.k) + layer * a.cache.layer;
  uint32_t* scales = (values ? a.cache.v_scales : a.cache.k_scales) + layer * a.cache.scale_layer;
  const int lane = threadIdx.x & (a.lanes - 1), teams = kQuantThreads >> a.log_lanes, rows = n * a.heads;
  struct Row {
    int t, h, node;
    piece p[WIDE ? N : 1];
  };
  auto head_of = [&](const Row& r) { return src + r.node * from.token_stride + r.h * from.head_stride; };
  auto load = [&](Row& r, int u) {
    if constexpr (WIDE)
#pragma unroll
      for (int j = 0; j < N; ++j) r.p[j] = *reinterpret_cast<const piece*>(head_of(r) + u * E + j * P);
  };
  auto find = [&](int i) {
    Row r;
    r.node = -1;
    if (i >= rows) return r;
    r.t = a.by_heads.of(i);
    r.h = i - r.t * a.heads;
    r.node = nodes[r.t];
    if (ONE && r.node >= 0 && lane < a.units) load(r, lane);
    return r;
  };
  Row next = find(threadIdx.x >> a.log_lanes);
  for (int i = threadIdx.x >> a.log_lanes; i < rows; i += teams) {
    Row row = next;
    next = find(i + teams);      // on its way meanwhile
    if (row.node < 0) continue;
    float x[E];
    auto take = [&](int u) {
      if (!ONE) load(row, u);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if constexpr (WIDE)
          x[e] = (float)row.p[e / P][e % P];
        else
          x[e] = (float)head_of(row)[min(u * E + e, a.head_dim - 1)];      // (the last element again changes no extent)
      }
    };
    Extent extent{0.f, INFINITY, -INFINITY};
    for (int u = lane; u < a.units; u += a.lanes) {
      take(u);
      extend<FORMAT, E>(extent, x);
    }
    if (FORMAT == kInt4) {
      extent.lo = team_all(extent.lo, a.lanes, [](float p, float q) { return least_of(p, p, q); });
      extent.hi = team_all(extent.hi, a.lanes, [](float p, float q) { return most_of(p, p, q); });
    } else {
      extent.most = team_all(extent.most, a.lanes, [](float p, float q) { return most_of(p, p, q); });
    }
    const Coder c = coder_of<FORMAT>(extent);
    if (lane == 0) scales[places[row.t][1] + row.h * a.cache.scale_head] = c.word;
    char* to = codes + places[row.t][0] + row.h * a.cache.head;
    for (int u = lane; u < a.units; u += a.lanes) {
      if (!ONE) take(u);
      uint32_t w[W];
      codes_of<FORMAT, E>(c, x, w);
      if constexpr (!WIDE) {
        const int bytes = FORMAT == kInt4 ? min(2, a.head_dim / 2 - 2 * u) : min(4, a.head_dim - 4 * u);
        for (int i = 0; i < bytes; ++i) to[u * (FORMAT == kInt4 ? 2 : 4) + i] = (char)(w[0] >> (8 * i));
      } else if constexpr (FORMAT == kInt4 && E == 4) {
        *reinterpret_cast<uint16_t*>(to + 2 * u) = (uint16_t)w[0];
      } else if constexpr (W == 1) {
        *reinterpret_cast<uint32_t*>(to + 4 * u) = w[0];
      } else if constexpr (W == 2) {
        *reinterpret_cast<uint2*>(to + 8 * u) = make_uint2(w[0], w[1]);
      } else {
        *reinterpret_cast<u32x4*>(to + 16 * u) = u32x4{w[0], w[1], w[2], w[3]};
      }
    }
  }
}

// ---- read ----
struct DequantizeArgs {
  QuantizedView cache;           // the first layer read
  Heads k, v;                    // [layers][batch][tokens][heads][head_dim]
  int64_t k_layer, v_layer;
  const int32_t *first, *count;
  Divide by_span, by_head;       // units of a head
  int tokens, head_dim, units, head_units, at_a_time, span, tokens_at_once;      // units of a token, of a head; units of a token and tokens that a workgroup takes at once
};
constexpr int kReadAtOnce = 4;      // tokens that a thread has on their way

// A workgroup makes at_a_time tokens of a layer of a sequence, keys or values; it looks their places up first.  A thread makes units of E elements, kReadAtOnce of them side by side.  What the cache
// does not hold is written as zeros.
template <int FORMAT, typename T, bool WIDE>
__global__ void __launch_bounds__(kQuantThreads) quantized_read_kernel(const DequantizeArgs a) {
  constexpr int E = WIDE ? Piece<T>::E : 4, W = E / 4;
  typedef typename Piece<T>::type piece;
  __shared__ int64_t places[kQuantTokens][2];      // -1: nothing is held
  const int b = blockIdx.z, layer = blockIdx.y >> 1, first = blockIdx.x * a.at_a_time;
  const bool values = blockIdx.y & 1;
  const Heads& into = values ? a.v : a.k;
  T* dst = reinterpret_cast<T*>(into.data) + layer * (values ? a.v_layer : a.k_layer) + b * into.batch_stride;
  const char* codes = (values ? a.cache.v : a.cache.k) + layer * a.cache.layer;
  const uint32_t* scales = (values ? a.cache.v_scales : a.cache.k_scales) + layer * a.cache.scale_layer;
  const int tokens = min(a.tokens - first, a.at_a_time);
  if ((int)threadIdx.x < tokens) {
    const int held = a.count == nullptr ? a.tokens : a.count[b];
    const int64_t place = (a.first == nullptr ? 0 : (int64_t)a.first[b]) + first + threadIdx.x;
    int64_t at = -1, scale_at = 0;
    if (first + (int)threadIdx.x >= held || place < 0 || place > 0x7fffffff || !a.cache.find(b, (uint32_t)place, &at, &scale_at)) at = -1;
    places[threadIdx.x][0] = at;
    places[threadIdx.x][1] = scale_at;
  }
  __syncthreads();
  // a thread has the same unit of every so many tokens (and every 256th, if a token has more), so that nothing is divided on the way
  const int t0 = a.by_span.of(threadIdx.x), each = a.tokens_at_once;
  if (t0 >= each) return;
  for (int u = (int)threadIdx.x - t0 * a.span; u < a.units; u += a.span) {
    const uint32_t h = a.by_head.of(u), e0 = (u - h * a.head_units) * E;
    const int64_t in_token = h * a.cache.head + (FORMAT == kInt4 ? e0 / 2 : e0), scale_in = h * a.cache.scale_head;
    T* out = dst + first * into.token_stride + h * into.head_stride + e0;
  for (int t = t0; t < tokens; t += kReadAtOnce * each) {
    struct Unit {
      uint32_t w[W], word;
      bool there;
    } x[kReadAtOnce];
#pragma unroll
    for (int k = 0; k < kReadAtOnce; ++k) {
      x[k] = Unit{};
      const int at_token = t + k * each;
      const int64_t at = at_token < tokens ? places[at_token][0] : -1;
      x[k].there = at >= 0;
      if (at < 0) continue;
      x[k].word = scales[places[at_token][1] + scale_in];
      const char* p = codes + at + in_token;
      if constexpr (!WIDE) {
        const int bytes = FORMAT == kInt4 ? min(2, (a.head_dim - (int)e0) / 2) : min(4, a.head_dim - (int)e0);
        for (int j = 0; j < bytes; ++j) x[k].w[0] |= (uint32_t)(uint8_t)p[j] << (8 * j);
      } else if constexpr (FORMAT == kInt4) {
        if constexpr (W == 1)
          x[k].w[0] = *reinterpret_cast<const uint16_t*>(p);
        else
          x[k].w[0] = *reinterpret_cast<const uint32_t*>(p);
      } else if constexpr (W == 1) {
        x[k].w[0] = *reinterpret_cast<const uint32_t*>(p);
      } else {
        const uint2 two = *reinterpret_cast<const uint2*>(p);
        x[k].w[0] = two.x;
        x[k].w[1] = two.y;
      }
    }
#pragma unroll
    for (int k = 0; k < kReadAtOnce; ++k) {
      if (t + k * each >= tokens) continue;
      uint32_t* w = x[k].w;
      if (FORMAT == kInt4) {
        if (W > 1) w[W - 1] = level_bytes<false>(apart(w[0] >> 16));
        w[0] = level_bytes<false>(apart(w[0] & 0xffffu));
      }
      float y[E];
#pragma unroll
      for (int j = 0; j < W; ++j) {
        float four[4];
        four_values<FORMAT>(w[j], x[k].word, four);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[4 * j + e] = x[k].there ? four[e] : 0.f;
      }
      T* to = out + (t + k * each) * into.token_stride;
      if constexpr (WIDE) {
        piece p;
#pragma unroll
        for (int e = 0; e < E; ++e) p[e] = (T)y[e];
        __builtin_nontemporal_store(p, reinterpret_cast<piece*>(to));
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if ((int)e0 + e < a.head_dim) to[e] = (T)y[e];
      }
    }
  }
  }
}

}  // namespace dpllm
