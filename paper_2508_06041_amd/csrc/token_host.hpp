// What the host side of the calls around the linears shares: the text of a refusal, checks and views of the caller's tensors.
#pragma once
#include <cstdarg>
#include <cstdio>

#include "token_common.hpp"

namespace dpllm {

// The text of the last refusal in this thread; a fixed array, so that nothing is allocated and nothing can throw.
char* call_error();
int refuse(int code, const char* format, ...) __attribute__((format(printf, 2, 3)));
int launched(const char* who);
// Errors of a cache as such, with `batch` sequences in it; 0: none.
int check_cache(const char* who, const dpllm_cache* cache, int batch);

// The same without the strides that no element is reached by: those of dimensions of 1 may be anything.
inline dpllm_heads reached(const dpllm_heads& t, int batch, int tokens, int heads) {
  return {t.data, batch > 1 ? t.batch_stride : 0, tokens > 1 ? t.token_stride : 0, heads > 1 ? t.head_stride : 0};
}
inline dpllm_cache reached(dpllm_cache c) {
  if (c.layers == 1) c.layer_stride = 0;
  if (c.pages == 1) c.page_stride = 0;
  if (c.page == 1) c.token_stride = 0;
  if (c.heads == 1) c.head_stride = 0;
  return c;
}

inline Heads view(const dpllm_heads& t) { return {(char*)t.data, t.batch_stride, t.token_stride, t.head_stride}; }

inline CacheView view(const dpllm_cache& c, int layer) {
  const int es = c.dtype == DPLLM_F32 ? 4 : 2;
  return {(char*)c.k + layer * c.layer_stride * es, (char*)c.v + layer * c.layer_stride * es, c.layer_stride, c.page_stride, c.token_stride,
          c.head_stride, c.table, c.table_stride, Divide::by(c.page), c.pages, c.page, c.pages_per_seq};
}

// whether 16 bytes of a head can be moved at a time
inline bool pieces(const dpllm_heads& t, int es) {
  return (uintptr_t)t.data % 16 == 0 && (t.batch_stride | t.token_stride | t.head_stride) % (16 / es) == 0;
}

}  // namespace dpllm
