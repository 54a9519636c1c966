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
// What a head's word takes: the largest size, as bits, so that NaN and infinity are larger than all else; of int4 the lowest and highest value too.
struct Extent {
  uint32_t most;
  float lo, hi;
};
__device__ __forceinline__ void extend(Extent& e, float x) {
  e.most = max(e.most, __float_as_uint(x) & 0x7fffffffu);
  e.lo = fminf(e.lo, x);
  e.hi = fmaxf(e.hi, x);
}
struct Coder {
  uint32_t word;
  float scale, offset, by, top;      // by: 1 / scale, or 127 / top
  bool flat, bad;                    // flat: all values are the offset
};
template <int FORMAT>
__device__ __forceinline__ Coder coder_of(const Extent& e) {
#pragma clang fp contract(off)
  Coder c{};
  c.bad = e.most >= 0x7f800000u;
  if (FORMAT == kInt4) {
    const float middle = e.lo * 0.5f + e.hi * 0.5f;
    const bfloat_t offset = (bfloat_t)middle;
    c.offset = (float)offset;
    const float reach = fmaxf(e.hi - c.offset, c.offset - e.lo);
    c.flat = !(reach > 0.f);
    const uint32_t up = (__float_as_uint(fmaxf(reach, kLeast) * 0.125f) + 0xffffu) & 0xffff0000u;
    c.scale = __uint_as_float(up);
    c.by = 1.0f / c.scale;
    c.bad = c.bad || up >= 0x7f800000u || (__float_as_uint(c.offset) & 0x7fffffffu) >= 0x7f800000u;
    c.word = c.bad ? kNan32 >> 16 : (c.flat ? 0u : up >> 16) | __float_as_uint(c.offset);
  } else {
    c.top = fmaxf(__uint_as_float(e.most), kLeast);
    if (FORMAT == kInt8) {
      c.scale = c.top / 127.0f;
      c.by = 127.0f / c.top;
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

// Four values as codes (of int4 nibbles in the lower bits of bytes).  The quotients of int8 and int4 are products with the reciprocal, and where one lands within 2^-14 of a border
// they are formed again as quotients: a product is off by 2^-23 of itself, of 127 at most, so the codes are those of quotients rounded once.
template <int FORMAT>
__device__ __forceinline__ uint32_t four_codes(const Coder& c, const float (&x)[4]) {
#pragma clang fp contract(off)
  uint32_t w = 0;
  if (c.bad) return 0u;
  if constexpr (FORMAT == kE4m3) {
    w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[0] * c.by, x[1] * c.by, 0, false);
    w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * c.by, x[3] * c.by, (int)w, true);
  } else if constexpr (FORMAT == kInt8) {
    float n[4], off = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float t = x[i] * c.by;
      n[i] = __builtin_rintf(t);
      off = fmaxf(off, __builtin_fabsf(t - n[i]));
    }
    if (off > 0.5f - 0x1p-14f) {
      const float down = c.top > 0x1p100f ? 0x1p-20f : 1.f;      // 127 x stays a float
#pragma unroll
      for (int i = 0; i < 4; ++i) n[i] = __builtin_rintf(x[i] * down * 127.0f / (c.top * down));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t)(int)n[i] & 0xffu) << (8 * i);
  } else {
    float n[4], low = 1.f, high = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float t = (x[i] - c.offset) * c.by;
      n[i] = __builtin_floorf(t);
      low = fminf(low, t - n[i]);
      high = fmaxf(high, t - n[i]);
    }
    if (low < 0x1p-14f || high > 1.f - 0x1p-14f)
#pragma unroll
      for (int i = 0; i < 4; ++i) n[i] = __builtin_floorf((x[i] - c.offset) / c.scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int level = (int)fminf(fmaxf(n[i], -8.f), 7.f);
      w |= (uint32_t)(level < 0 ? 7 - level : level) << (8 * i);      // 8 + (-1 - level)
    }
  }
  return w;
}
// Four nibbles of four bytes, side by side.
__device__ __forceinline__ uint32_t side_by_side(uint32_t w) {
  w |= w >> 4;      // bytes 0 and 2 hold two codes each
  return (w & 0xffu) | ((w >> 8) & 0xff00u);
}
__device__ __forceinline__ uint32_t apart(uint32_t w) {      // back: 16 bits to four bytes
  w = (w & 0xffu) | ((w & 0xff00u) << 8);
  return (w & 0x000f000fu) | ((w & 0x00f000f0u) << 4);
}

// ---- append ----
constexpr int kQuantThreads = 256;

struct QuantizeArgs {
  QuantizedView cache;           // the first layer written
  Heads k, v;                    // [layers][batch][tokens][heads][head_dim]
  int64_t k_layer, v_layer;
  const int32_t *lens, *path, *count;
  int64_t path_stride;
  Divide by_heads;
  int tokens, heads, head_dim, units, lanes, log_lanes, at_a_time;      // units of E elements to a head, lanes that share one
};

// A group of `lanes` lanes (a power of two) quantises a head of a token: its values are read once into registers where there are no more units than lanes (ONE), else twice.
// Grid: (sequence, 2 layers + (keys, values), at_a_time tokens).  A unit is E elements; without WIDE it is read and written element by element, and the last may be short.
// Bound by the latency of a launch for single tokens, by memory for prompts.
template <int FORMAT, typename T, bool WIDE, bool ONE>
__global__ void __launch_bounds__(kQuantThreads) quantized_append_kernel(const QuantizeArgs a) {
  constexpr int E = WIDE ? Piece<T>::E : 4, W = E / 4;
  typedef typename Piece<T>::type piece;
  const int b = blockIdx.x, layer = blockIdx.y >> 1, first = blockIdx.z * a.at_a_time;
  const bool values = blockIdx.y & 1;
  int n = a.count == nullptr ? a.tokens : min(a.count[b], a.tokens);
  n = min(n - first, a.at_a_time);
  if (n <= 0) return;
  const int base = a.lens[b];
  if (base < 0) return;
  const Heads& from = values ? a.v : a.k;
  const T* src = reinterpret_cast<const T*>(from.data) + layer * (values ? a.v_layer : a.k_layer) + b * from.batch_stride;
  char* codes = (values ? a.cache.v : a.cache.k) + layer * a.cache.layer;
  uint32_t* scales = (values ? a.cache.v_scales : a.cache.k_scales) + layer * a.cache.scale_layer;
  const int lane = threadIdx.x & (a.lanes - 1), teams = kQuantThreads >> a.log_lanes;
  for (int i = threadIdx.x >> a.log_lanes; i < n * a.heads; i += teams) {
    const uint32_t t = a.by_heads.of(i), h = i - t * a.heads, place = first + t;
    const int node = a.path == nullptr ? (int)place : a.path[b * a.path_stride + place];
    int64_t at, scale_at;
    if ((uint32_t)node >= (uint32_t)a.tokens || (uint32_t)base + place > 0x7fffffffu || !a.cache.find(b, (uint32_t)base + place, &at, &scale_at)) continue;
    const T* head = src + node * from.token_stride + h * from.head_stride;
    float x[E];
    auto load = [&](int u) {
      if constexpr (WIDE) {
        const piece p = *reinterpret_cast<const piece*>(head + u * E);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = (float)p[e];
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = (float)head[min(u * E + e, a.head_dim - 1)];      // (the last element again changes no extent)
      }
    };
    Extent extent{0u, INFINITY, -INFINITY};
    for (int u = lane; u < a.units; u += a.lanes) {
      load(u);
#pragma unroll
      for (int e = 0; e < E; ++e) extend(extent, x[e]);
    }
    extent.most = team_all(extent.most, a.lanes, [](uint32_t p, uint32_t q) { return max(p, q); });
    if (FORMAT == kInt4) {
      extent.lo = team_all(extent.lo, a.lanes, [](float p, float q) { return fminf(p, q); });
      extent.hi = team_all(extent.hi, a.lanes, [](float p, float q) { return fmaxf(p, q); });
    }
    const Coder c = coder_of<FORMAT>(extent);
    if (lane == 0) scales[scale_at + h * a.cache.scale_head] = c.word;
    char* to = codes + at + h * a.cache.head;
    for (int u = lane; u < a.units; u += a.lanes) {
      if (!ONE) load(u);
      uint32_t w[W];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float four[4] = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
        w[i] = four_codes<FORMAT>(c, four);
        if (FORMAT == kInt4) w[i] = side_by_side(w[i]);
      }
      if constexpr (!WIDE) {
        const int bytes = FORMAT == kInt4 ? min(2, a.head_dim / 2 - 2 * u) : min(4, a.head_dim - 4 * u);
        for (int i = 0; i < bytes; ++i) to[u * (FORMAT == kInt4 ? 2 : 4) + i] = (char)(w[0] >> (8 * i));
      } else if constexpr (FORMAT == kInt4) {
        if constexpr (W == 1)
          *reinterpret_cast<uint16_t*>(to + 2 * u) = (uint16_t)w[0];
        else
          *reinterpret_cast<uint32_t*>(to + 4 * u) = w[0] | w[1] << 16;
      } else if constexpr (W == 1) {
        *reinterpret_cast<uint32_t*>(to + 4 * u) = w[0];
      } else {
        *reinterpret_cast<uint2*>(to + 8 * u) = make_uint2(w[0], w[1]);
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
  Divide by_units, by_head;      // units of a token, of a head
  int tokens, head_dim, units, head_units, at_a_time;
};

// A thread makes a unit of E elements; grid as above.  What the cache does not hold is written as zeros.
template <int FORMAT, typename T, bool WIDE>
__global__ void __launch_bounds__(kQuantThreads) quantized_read_kernel(const DequantizeArgs a) {
  constexpr int E = WIDE ? Piece<T>::E : 4, W = E / 4;
  typedef typename Piece<T>::type piece;
  const int b = blockIdx.x, layer = blockIdx.y >> 1, first = blockIdx.z * a.at_a_time;
  const bool values = blockIdx.y & 1;
  const Heads& into = values ? a.v : a.k;
  T* dst = reinterpret_cast<T*>(into.data) + layer * (values ? a.v_layer : a.k_layer) + b * into.batch_stride;
  const char* codes = (values ? a.cache.v : a.cache.k) + layer * a.cache.layer;
  const uint32_t* scales = (values ? a.cache.v_scales : a.cache.k_scales) + layer * a.cache.scale_layer;
  const int64_t from = a.first == nullptr ? 0 : a.first[b];
  const int held = a.count == nullptr ? a.tokens : a.count[b];
  const uint32_t end = (uint32_t)min(a.tokens - first, a.at_a_time) * a.units;
  for (uint32_t i = threadIdx.x; i < end; i += kQuantThreads) {
    const uint32_t t = a.by_units.of(i), u = i - t * a.units, h = a.by_head.of(u), e0 = (u - h * a.head_units) * E;
    const int64_t place = from + first + t;
    int64_t at, scale_at;
    uint32_t w[W] = {}, word = 0;
    const bool there = (int)(first + t) < held && place >= 0 && place <= 0x7fffffff && a.cache.find(b, (uint32_t)place, &at, &scale_at);
    if (there) {
      word = scales[scale_at + h * a.cache.scale_head];
      const char* p = codes + at + h * a.cache.head + (FORMAT == kInt4 ? e0 / 2 : e0);
      if constexpr (!WIDE) {
        const int bytes = FORMAT == kInt4 ? min(2, (a.head_dim - (int)e0) / 2) : min(4, a.head_dim - (int)e0);
        for (int j = 0; j < bytes; ++j) w[0] |= (uint32_t)(uint8_t)p[j] << (8 * j);
      } else if constexpr (FORMAT == kInt4) {
        if constexpr (W == 1)
          w[0] = *reinterpret_cast<const uint16_t*>(p);
        else
          w[0] = *reinterpret_cast<const uint32_t*>(p);
      } else {
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
      }
    }
    if (FORMAT == kInt4) {
      if (W > 1) w[W - 1] = level_bytes<false>(apart(w[0] >> 16));
      w[0] = level_bytes<false>(apart(w[0] & 0xffffu));
    }
    float x[E];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      float four[4];
      four_values<FORMAT>(w[j], word, four);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * j + e] = there ? four[e] : 0.f;
    }
    T* to = dst + (first + t) * into.token_stride + h * into.head_stride + e0;
    if constexpr (WIDE) {
      piece p;
#pragma unroll
      for (int e = 0; e < E; ++e) p[e] = (T)x[e];
      *reinterpret_cast<piece*>(to) = p;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if ((int)e0 + e < a.head_dim) to[e] = (T)x[e];
    }
  }
}

}  // namespace dpllm
