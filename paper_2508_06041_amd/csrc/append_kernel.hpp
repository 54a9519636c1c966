// Keys and values of the tokens that stand go into the pages of the cache, for several layers at once.
#pragma once
#include "token_common.hpp"

namespace dpllm {

constexpr int kAppendThreads = 256;
constexpr int kAppendAtOnce = 2;      // pieces of keys and of values that a thread has on their way (55 MB: 2 7.0 us, 4 8.2)

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
// Bound by memory and the latency of a launch: 55 MB (read and written) of 48 layers in 7 us, 7.8 TB/s with some of it in the caches.
template <typename T>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendArgs a, int elements) {
  const int b = blockIdx.x, layer = blockIdx.y, first = blockIdx.z * a.at_a_time;
  int n = a.count == nullptr ? a.tokens : min(a.count[b], a.tokens);
  n = min(n - first, a.at_a_time);
  if (n <= 0) return;
  const int base = a.lens[b];
  if (base < 0) return;
  const int es = (int)(sizeof(T) / elements);
  const char *src_k = a.k.data + (layer * a.k_layer + b * a.k.batch_stride) * es, *src_v = a.v.data + (layer * a.v_layer + b * a.v.batch_stride) * es;
  const uint32_t end = (uint32_t)n * a.units;
  for (uint32_t start = threadIdx.x; start < end; start += kAppendAtOnce * kAppendThreads) {
    T k[kAppendAtOnce], v[kAppendAtOnce];
    int64_t to[kAppendAtOnce];
#pragma unroll
    for (int j = 0; j < kAppendAtOnce; ++j) {
      const uint32_t i = start + j * kAppendThreads;
      to[j] = -1;
      if (i >= end) continue;
      const uint32_t t = a.by_units.of(i), u = i - t * a.units, h = a.by_head.of(u), e = (u - h * a.head_units) * elements;
      const uint32_t place = first + t;
      const int from = a.path == nullptr ? (int)place : a.path[b * a.path_stride + place];
      int64_t at;
      if ((uint32_t)from >= (uint32_t)a.tokens || (uint32_t)base + place > 0x7fffffffu || !a.cache.find(b, (uint32_t)base + place, &at)) continue;
      to[j] = (at + layer * a.cache.layer_stride + h * a.cache.head_stride + e) * es;
      k[j] = *reinterpret_cast<const T*>(src_k + (from * a.k.token_stride + h * a.k.head_stride + e) * es);
      v[j] = *reinterpret_cast<const T*>(src_v + (from * a.v.token_stride + h * a.v.head_stride + e) * es);
    }
#pragma unroll
    for (int j = 0; j < kAppendAtOnce; ++j) {
      if (to[j] < 0) continue;
      *reinterpret_cast<T*>(a.cache.k + to[j]) = k[j];
      *reinterpret_cast<T*>(a.cache.v + to[j]) = v[j];
    }
  }
}

}  // namespace dpllm
