// Keys and values of the tokens that stand go into the pages of the cache, for several layers at once.
#pragma once
#include "token_common.hpp"

namespace dpllm {

constexpr int kAppendThreads = 256;

struct AppendArgs {
  CacheView cache;               // k, v: the first layer written
  Heads k, v;                    // [layers][batch][tokens][heads][head_dim]
  int64_t k_layer, v_layer;
  const int32_t *lens, *path, *count;
  int64_t path_stride;
  Divide by_units, by_head;      // pieces of a token, of a head
  int batch, tokens, units, head_units, at_a_time;
};

// A workgroup copies up to at_a_time tokens of one layer of one sequence, keys and values; how many there are it learns on the device.  A piece is
// 16 bytes, or one element (T) where the layout does not allow that.  The nodes' own tensors are only read, so the order does not matter
// and a second call with the same arguments changes nothing.
template <typename T>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendArgs a, int elements) {
  const int b = blockIdx.x, layer = blockIdx.y, first = blockIdx.z * a.at_a_time;
  int n = a.count == nullptr ? a.tokens : min(a.count[b], a.tokens);
  n = min(n - first, a.at_a_time);
  if (n <= 0) return;
  const int base = a.lens[b];
  if (base < 0) return;
  const char *src_k = a.k.data + (layer * a.k_layer + b * a.k.batch_stride) * (int64_t)(sizeof(T) / elements),
             *src_v = a.v.data + (layer * a.v_layer + b * a.v.batch_stride) * (int64_t)(sizeof(T) / elements);
  const int es = (int)(sizeof(T) / elements);
  for (uint32_t i = threadIdx.x; i < (uint32_t)n * a.units; i += kAppendThreads) {
    const uint32_t t = a.by_units.of(i), u = i - t * a.units, h = a.by_head.of(u), e = (u - h * a.head_units) * elements;
    const uint32_t place = first + t;
    const int from = a.path == nullptr ? (int)place : a.path[b * a.path_stride + place];
    int64_t at;
    if ((uint32_t)from >= (uint32_t)a.tokens || (uint32_t)base + place > 0x7fffffffu || !a.cache.find(b, (uint32_t)base + place, &at)) continue;
    at += layer * a.cache.layer_stride + h * a.cache.head_stride + e;
    const T k = *reinterpret_cast<const T*>(src_k + (from * a.k.token_stride + h * a.k.head_stride + e) * es);
    const T v = *reinterpret_cast<const T*>(src_v + (from * a.v.token_stride + h * a.v.head_stride + e) * es);
    *reinterpret_cast<T*>(a.cache.k + at * es) = k;
    *reinterpret_cast<T*>(a.cache.v + at * es) = v;
  }
}

}  // namespace dpllm
