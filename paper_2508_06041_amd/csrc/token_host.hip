// See token_host.hpp.
#include "token_host.hpp"

namespace dpllm {

char* call_error() {
  static thread_local char text[256] = "";
  return text;
}

int refuse(int code, const char* format, ...) {
  va_list args;
  va_start(args, format);
  vsnprintf(call_error(), 256, format, args);
  va_end(args);
  return code;
}

int launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? DPLLM_OK : refuse(DPLLM_EHIP, "%s: %s", who, hipGetErrorString(e));
}

int check_cache(const char* who, const dpllm_cache* c, int batch) {
  if (!c || !c->k || !c->v) return refuse(DPLLM_EINVAL, "%s: the cache, its k or its v is NULL", who);
  if (c->dtype < DPLLM_F16 || c->dtype > DPLLM_F32) return refuse(DPLLM_EINVAL, "%s: unknown dtype %d", who, c->dtype);
  if (c->layers < 1 || c->pages < 1 || c->page < 1 || c->pages_per_seq < 1 || c->heads < 1 || c->head_dim < 1 || c->head_dim > DPLLM_MAX_HEAD_DIM ||
      (int64_t)c->heads * c->head_dim > (1 << 24))
    return refuse(DPLLM_ESHAPE, "%s: a cache of %d layers, %d pages of %d tokens, %d to a sequence, %d heads of %d", who, c->layers, c->pages, c->page,
                  c->pages_per_seq, c->heads, c->head_dim);
  if (((uintptr_t)c->k | (uintptr_t)c->v) % (c->dtype == DPLLM_F32 ? 4 : 2)) return refuse(DPLLM_EINVAL, "%s: the cache is not aligned to its elements", who);
  if (!c->table && (c->pages_per_seq != 1 || batch > c->pages))
    return refuse(DPLLM_ESHAPE, "%s: a cache without a table has one page per sequence (%d pages for %d sequences)", who, c->pages, batch);
  if (c->table && c->table_stride < 0) return refuse(DPLLM_ESHAPE, "%s: negative table_stride", who);
  return DPLLM_OK;
}

}  // namespace dpllm
