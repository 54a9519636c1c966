// Host side of dpllm_tree_attention: argument checks, how the work is split, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "attention_plan.hpp"
#include "token_host.hpp"
#include "tree_attention.hpp"

using namespace dpllm;

namespace {

template <typename T, int D>
void launch(const AttentionArgs& a, const AttentionPlan& p, hipStream_t s) {
  const dim3 groups((unsigned)p.groups);
  if constexpr (D == 64 || D == 128)
    if (p.lone) hipLaunchKernelGGL((tree_attention_kernel<T, D, 1, 8>), groups, dim3(8 * 64), 0, s, a);
  if (p.waves == 0 && p.mt == 1 && !p.lone) hipLaunchKernelGGL((tree_attention_kernel<T, D, 1, kAttWaves>), groups, dim3(kAttWaves * 64), 0, s, a);
  if (p.waves == 4 && p.mt == 1) hipLaunchKernelGGL((tree_attention_wide_kernel<T, D, 1, 4>), groups, dim3(4 * 64), 0, s, a);
  if constexpr (D < 256) {
    if (p.waves == 0 && p.mt == 2) hipLaunchKernelGGL((tree_attention_kernel<T, D, 2, kAttWaves>), groups, dim3(kAttWaves * 64), 0, s, a);
    if (p.waves == 4 && p.mt == 2) hipLaunchKernelGGL((tree_attention_wide_kernel<T, D, 2, 4>), groups, dim3(4 * 64), 0, s, a);
    if (p.waves == 8 && p.mt == 2) hipLaunchKernelGGL((tree_attention_wide_kernel<T, D, 2, 8>), groups, dim3(8 * 64), 0, s, a);
  }
  if (p.bytes > 0) {
    const uint32_t all_rows = (uint32_t)a.batch * a.kv_heads * a.rows;
    hipLaunchKernelGGL((tree_attention_join_kernel<T, D>), dim3((all_rows + 3) / 4), dim3(256), 0, s, a, p.tile, Divide::by(a.rows), Divide::by(a.kv_heads),
                       Divide::by(p.tile), all_rows);
  }
}

template <typename T>
void launch(int head_dim, const AttentionArgs& a, const AttentionPlan& p, hipStream_t s) {
  if (head_dim == 64) launch<T, 64>(a, p, s);
  if (head_dim == 96) launch<T, 96>(a, p, s);
  if (head_dim == 128) launch<T, 128>(a, p, s);
  if (head_dim == 256) launch<T, 256>(a, p, s);
}

}  // namespace

extern "C" {

int dpllm_tree_attention_workspace_bytes(int batch, int nodes, int heads, int kv_heads, int head_dim, int max_len, size_t* bytes) {
  const char* who = "dpllm_tree_attention_workspace_bytes";
  if (!bytes) return refuse(DPLLM_EINVAL, "%s: bytes is NULL", who);
  if (int rc = check_attention(who, batch, nodes, heads, kv_heads, head_dim)) return rc;
  if (max_len < 0) return refuse(DPLLM_ESHAPE, "%s: max_len %d", who, max_len);
  *bytes = batch == 0 || nodes == 0 ? 0 : plan_attention(batch, nodes, heads, kv_heads, head_dim, max_len).bytes;
  return DPLLM_OK;
}

int dpllm_tree_attention(const dpllm_cache* cache, int layer, int batch, int nodes, int heads, const int32_t* lens_dev, int max_len,
                         const dpllm_heads* q, const dpllm_heads* k_new, const dpllm_heads* v_new, const uint64_t* mask_dev, int64_t mask_stride,
                         float scale, const dpllm_heads* out, float* lse_dev, void* ws_dev, size_t ws_bytes, void* stream) {
  const char* who = "dpllm_tree_attention";
  if (int rc = check_cache(who, cache, batch)) return rc;
  if (cache->dtype == DPLLM_F32) return refuse(DPLLM_EINVAL, "%s: takes float16 and bfloat16", who);
  if (int rc = check_attention(who, batch, nodes, heads, cache->heads, cache->head_dim)) return rc;
  if (layer < 0 || layer >= cache->layers) return refuse(DPLLM_ERANGE, "%s: layer %d of %d", who, layer, cache->layers);
  if (max_len < 0) return refuse(DPLLM_ESHAPE, "%s: max_len %d", who, max_len);
  if ((int64_t)cache->pages_per_seq * cache->page > INT32_MAX - 256) return refuse(DPLLM_ESHAPE, "%s: more than 2^31 - 256 tokens to a sequence", who);
  if (!std::isfinite(scale)) return refuse(DPLLM_EINVAL, "%s: scale is not finite", who);
  if (batch == 0 || nodes == 0) return DPLLM_OK;
  if (!lens_dev || !q || !out || !q->data || !out->data || !k_new != !v_new || (k_new && (!k_new->data || !v_new->data)))
    return refuse(DPLLM_EINVAL, "%s: a pointer is NULL (k_new and v_new may be, together)", who);
  const dpllm_cache c = reached(*cache);
  const dpllm_heads queries = reached(*q, batch, nodes, heads), results = reached(*out, batch, nodes, heads);
  const dpllm_heads keys = k_new ? reached(*k_new, batch, nodes, c.heads) : dpllm_heads{}, values = k_new ? reached(*v_new, batch, nodes, c.heads) : dpllm_heads{};
  if (!pieces(queries, 2) || !pieces(results, 2) || !pieces(keys, 2) || !pieces(values, 2) || ((uintptr_t)c.k | (uintptr_t)c.v) % 16 ||
      (c.layer_stride | c.page_stride | c.token_stride | c.head_stride) % 8)
    return refuse(DPLLM_EINVAL, "%s: tensors have to be aligned to 16 bytes, with strides of whole 8 elements", who);
  const AttentionPlan p = plan_attention(batch, nodes, heads, cache->heads, cache->head_dim, std::min<int64_t>(max_len, (int64_t)cache->pages_per_seq * cache->page));
  if (p.groups > 0x7fffff || (int64_t)batch * heads * nodes > 0x7fffff) return refuse(DPLLM_ESHAPE, "%s: %lld workgroups", who, (long long)p.groups);
  if (p.bytes > 0 && (!ws_dev || ws_bytes < p.bytes || (uintptr_t)ws_dev % 16))
    return refuse(DPLLM_ESTATE, "%s: needs a workspace of %zu bytes, aligned to 16", who, p.bytes);
  AttentionArgs a{};
  a.cache = view(c, layer);
  a.q = view(queries);
  a.out = view(results);
  a.k_new = view(keys);
  a.v_new = view(values);
  a.lens = lens_dev;
  a.mask = mask_dev;
  a.mask_stride = mask_stride;
  a.lse = lse_dev;
  place_workspace(a, p, ws_dev);
  fill_attention(a, p, batch, nodes, heads, cache->heads, k_new != nullptr, scale);
  if (cache->dtype == DPLLM_F16)
    launch<half_t>(cache->head_dim, a, p, (hipStream_t)stream);
  else
    launch<bfloat_t>(cache->head_dim, a, p, (hipStream_t)stream);
  return launched(who);
}

}  // extern "C"
