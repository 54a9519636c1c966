// What the kernels around the linears share: element types, 128-bit pieces of a tensor, tokens of a paged cache.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/dpllm.h"

namespace dpllm {

typedef _Float16 half_t;
typedef __bf16 bfloat_t;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of a tensor as E elements
template <typename T>
struct Piece {
  static constexpr int E = 16 / sizeof(T);
  typedef T type __attribute__((ext_vector_type(E)));
};

// A tensor [batch][tokens][heads][head_dim], strides in elements.
struct Heads {
  char* data;
  int64_t batch_stride, token_stride, head_stride;
};

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31 without a division: n * mul >> (32 + shift), mul = floor(2^(32 + shift) / d) + 1 with
// 2^(shift + 1) >= d > 2^shift, exact because mul * d exceeds 2^(32 + shift) by at most d <= 2^(shift + 1), so by less than 2^(32 + shift) / n.
// Powers of two (and 1) have mul = 0 and only shift.
struct Divide {
  uint32_t mul;
  int shift;
  static Divide by(uint32_t d) {
    int s = 0;
    while (s < 31 && (2ull << s) <= d) ++s;   // 2^s <= d < 2^(s + 1)
    if ((d & (d - 1)) == 0) return {0u, s};
    return {(uint32_t)((1ull << (32 + s)) / d + 1), s};
  }
  __device__ __forceinline__ uint32_t of(uint32_t n) const { return mul == 0 ? n >> shift : __umulhi(n, mul) >> shift; }
};

// The keys and values of one layer of a paged cache, as kernels read and write them.
struct CacheView {
  char *k, *v;
  int64_t layer_stride, page_stride, token_stride, head_stride;   // elements
  const int32_t* table;                                           // [batch][table_stride], nullptr: sequence b has page b
  int64_t table_stride;
  Divide by_page;
  int pages, page, pages_per_seq;
  // Where token t of sequence b starts, in elements; false: no page holds it (an id out of the pool, or past the table).
  __device__ __forceinline__ bool find(int b, uint32_t t, int64_t* at) const {
    const uint32_t j = by_page.of(t);
    if (j >= (uint32_t)pages_per_seq) return false;
    const int id = table == nullptr ? b : table[b * table_stride + j];
    if ((uint32_t)id >= (uint32_t)pages) return false;
    *at = (int64_t)id * page_stride + (int64_t)(t - j * (uint32_t)page) * token_stride;
    return true;
  }
};

}  // namespace dpllm
