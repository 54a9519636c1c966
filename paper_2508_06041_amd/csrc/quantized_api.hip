// Host side of the calls on a quantised cache that include/dpllm.h declares: argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "quantized_launch.hpp"
#include "token_host.hpp"

using namespace dpllm;

namespace dpllm {
template <>
void launch_quantized<kE4m3>(int, int, const QuantizedArgs&, const QuantizedPlan&, hipStream_t);
template <>
void launch_quantized<kInt8>(int, int, const QuantizedArgs&, const QuantizedPlan&, hipStream_t);
template <>
void launch_quantized<kInt4>(int, int, const QuantizedArgs&, const QuantizedPlan&, hipStream_t);
}  // namespace dpllm

namespace {

int check_quantized(const char* who, const dpllm_quantized_cache* c, int batch) {
  if (!c || !c->k || !c->v || !c->k_scales || !c->v_scales) return refuse(DPLLM_EINVAL, "%s: the cache, its codes or its scales are NULL", who);
  if (c->format < DPLLM_CACHE_E4M3 || c->format > DPLLM_CACHE_INT4) return refuse(DPLLM_EINVAL, "%s: unknown format %d", who, c->format);
  if (c->layers < 1 || c->pages < 1 || c->page < 1 || c->pages_per_seq < 1 || c->heads < 1 || c->head_dim < 1 || c->head_dim > DPLLM_MAX_HEAD_DIM ||
      (int64_t)c->heads * c->head_dim > (1 << 24))
    return refuse(DPLLM_ESHAPE, "%s: a cache of %d layers, %d pages of %d tokens, %d to a sequence, %d heads of %d", who, c->layers, c->pages, c->page,
                  c->pages_per_seq, c->heads, c->head_dim);
  if (c->format == DPLLM_CACHE_INT4 && c->head_dim % 2) return refuse(DPLLM_ESHAPE, "%s: head_dim %d is odd, which INT4 does not hold", who, c->head_dim);
  if (((uintptr_t)c->k_scales | (uintptr_t)c->v_scales) % 4) return refuse(DPLLM_EINVAL, "%s: the scales are not aligned to their words", who);
  if (!c->table && (c->pages_per_seq != 1 || batch > c->pages))
    return refuse(DPLLM_ESHAPE, "%s: a cache without a table has one page per sequence (%d pages for %d sequences)", who, c->pages, batch);
  if (c->table && c->table_stride < 0) return refuse(DPLLM_ESHAPE, "%s: negative table_stride", who);
  return DPLLM_OK;
}

// The strides that no element is reached by count as 0.
dpllm_quantized_cache reached(dpllm_quantized_cache c) {
  if (c.layers == 1) c.layer_stride = c.scale_layer_stride = 0;
  if (c.pages == 1) c.page_stride = c.scale_page_stride = 0;
  if (c.page == 1) c.token_stride = c.scale_token_stride = 0;
  if (c.heads == 1) c.head_stride = c.scale_head_stride = 0;
  return c;
}

QuantizedView view(const dpllm_quantized_cache& c, int layer) {
  return {(char*)c.k + layer * c.layer_stride, (char*)c.v + layer * c.layer_stride, (uint32_t*)c.k_scales + layer * c.scale_layer_stride,
          (uint32_t*)c.v_scales + layer * c.scale_layer_stride, c.layer_stride, c.page_stride, c.token_stride, c.head_stride, c.scale_layer_stride, c.scale_page_stride,
          c.scale_token_stride, c.scale_head_stride, c.table, c.table_stride, Divide::by(c.page), c.pages, c.page, c.pages_per_seq};
}

// whether the codes of so many elements can be moved at a time
bool whole_codes(const dpllm_quantized_cache& c, int elements) {
  const int bytes = c.format == DPLLM_CACHE_INT4 ? elements / 2 : elements;
  return ((uintptr_t)c.k | (uintptr_t)c.v) % bytes == 0 && (c.layer_stride | c.page_stride | c.token_stride | c.head_stride) % bytes == 0;
}

// f(format, type) with the constants that belong to the arguments
template <typename F>
void choose(int format, int dtype, F f) {
  auto by_type = [&](auto form) {
    if (dtype == DPLLM_F16) f(form, half_t());
    if (dtype == DPLLM_BF16) f(form, bfloat_t());
    if (dtype == DPLLM_F32) f(form, float());
  };
  if (format == kE4m3) by_type(std::integral_constant<int, kE4m3>());
  if (format == kInt8) by_type(std::integral_constant<int, kInt8>());
  if (format == kInt4) by_type(std::integral_constant<int, kInt4>());
}

// What append and read refuse alike.
int check_layers(const char* who, const dpllm_quantized_cache* cache, int first_layer, int n_layers, int batch, int tokens, int dtype, const dpllm_heads* k,
                 const dpllm_heads* v) {
  if (int rc = check_quantized(who, cache, batch)) return rc;
  if (!k || !v) return refuse(DPLLM_EINVAL, "%s: a pointer is NULL", who);
  if (dtype < DPLLM_F16 || dtype > DPLLM_F32) return refuse(DPLLM_EINVAL, "%s: unknown dtype %d", who, dtype);
  if (first_layer < 0 || n_layers < 0 || n_layers > cache->layers - first_layer || n_layers > 32767)
    return refuse(DPLLM_ERANGE, "%s: layers %d to %lld of %d", who, first_layer, (long long)first_layer + n_layers, cache->layers);
  if (batch < 0 || batch > 65535 || tokens < 0 || tokens > (1 << 24)) return refuse(DPLLM_ESHAPE, "%s: %d sequences of %d tokens (at most 65535 of 2^24)", who, batch, tokens);
  if (((uintptr_t)k->data | (uintptr_t)v->data) % (dtype == DPLLM_F32 ? 4 : 2)) return refuse(DPLLM_EINVAL, "%s: keys or values are not aligned to their elements", who);
  return DPLLM_OK;
}

}  // namespace

extern "C" {

int dpllm_quantized_append(const dpllm_quantized_cache* cache, int first_layer, int n_layers, int batch, int nodes, const int32_t* lens_dev, int dtype,
                           const dpllm_heads* k_new, int64_t k_layer_stride, const dpllm_heads* v_new, int64_t v_layer_stride, const int32_t* path_dev,
                           int64_t path_stride, const int32_t* count_dev, void* stream) {
  const char* who = "dpllm_quantized_append";
  if (int rc = check_layers(who, cache, first_layer, n_layers, batch, nodes, dtype, k_new, v_new)) return rc;
  if (!lens_dev && batch > 0) return refuse(DPLLM_EINVAL, "%s: a pointer is NULL", who);
  if (n_layers == 0 || batch == 0 || nodes == 0) return DPLLM_OK;
  if (!k_new->data || !v_new->data) return refuse(DPLLM_EINVAL, "%s: k_new or v_new is NULL", who);
  const int es = dtype == DPLLM_F32 ? 4 : 2, wide = 16 / es;
  const dpllm_quantized_cache c = reached(*cache);
  const dpllm_heads k = reached(*k_new, batch, nodes, c.heads), v = reached(*v_new, batch, nodes, c.heads);
  if (n_layers == 1) k_layer_stride = v_layer_stride = 0;
  const bool vector = c.head_dim % wide == 0 && pieces(k, es) && pieces(v, es) && (k_layer_stride | v_layer_stride) % wide == 0 && whole_codes(c, wide);
  QuantizeArgs a{};
  a.cache = view(c, first_layer);
  a.k = view(k);
  a.v = view(v);
  a.k_layer = k_layer_stride;
  a.v_layer = v_layer_stride;
  a.lens = lens_dev;
  a.path = path_dev;
  a.count = count_dev;
  a.path_stride = path_stride;
  a.by_heads = Divide::by(c.heads);
  a.tokens = nodes;
  a.heads = c.heads;
  a.head_dim = c.head_dim;
  const int pieces_each = !vector ? 0 : c.head_dim % (2 * wide) == 0 && whole_codes(c, 2 * wide) ? 2 : 1;
  const int e = vector ? pieces_each * wide : 4;
  a.units = (c.head_dim + e - 1) / e;
  while ((1 << a.log_lanes) < std::min(a.units, 64)) ++a.log_lanes;
  a.lanes = 1 << a.log_lanes;
  // as many tokens to a workgroup as leave eight workgroups to a compute unit, eight heads to a group of lanes at most
  const int teams = kQuantThreads >> a.log_lanes;
  const int64_t all = (int64_t)nodes * c.heads * batch * 2 * n_layers;
  const int per = std::max(1, (int)std::min<int64_t>(8, all / ((int64_t)teams * 2048)));
  a.at_a_time = std::max(1, std::min(kQuantTokens, per * teams / c.heads));
  const dim3 grid((nodes + a.at_a_time - 1) / a.at_a_time, 2 * n_layers, batch);
  choose(c.format, dtype, [&](auto form, auto type) {
    auto launch = [&](auto n, auto one) {
      hipLaunchKernelGGL((quantized_append_kernel<decltype(form)::value, decltype(type), decltype(n)::value, decltype(one)::value>), grid, dim3(kQuantThreads), 0,
                         (hipStream_t)stream, a);
    };
    auto by_one = [&](auto n) { a.units <= a.lanes ? launch(n, std::true_type()) : launch(n, std::false_type()); };
    if (pieces_each == 0) by_one(std::integral_constant<int, 0>());
    if (pieces_each == 1) by_one(std::integral_constant<int, 1>());
    if (pieces_each == 2) by_one(std::integral_constant<int, 2>());
  });
  return launched(who);
}

int dpllm_quantized_read(const dpllm_quantized_cache* cache, int first_layer, int n_layers, int batch, int tokens, const int32_t* first_dev, const int32_t* count_dev,
                         int dtype, const dpllm_heads* k_out, int64_t k_layer_stride, const dpllm_heads* v_out, int64_t v_layer_stride, void* stream) {
  const char* who = "dpllm_quantized_read";
  if (int rc = check_layers(who, cache, first_layer, n_layers, batch, tokens, dtype, k_out, v_out)) return rc;
  if (n_layers == 0 || batch == 0 || tokens == 0) return DPLLM_OK;
  if (!k_out->data || !v_out->data) return refuse(DPLLM_EINVAL, "%s: k_out or v_out is NULL", who);
  const int es = dtype == DPLLM_F32 ? 4 : 2, wide = 16 / es;
  const dpllm_quantized_cache c = reached(*cache);
  const dpllm_heads k = reached(*k_out, batch, tokens, c.heads), v = reached(*v_out, batch, tokens, c.heads);
  if (n_layers == 1) k_layer_stride = v_layer_stride = 0;
  const bool vector = c.head_dim % wide == 0 && pieces(k, es) && pieces(v, es) && (k_layer_stride | v_layer_stride) % wide == 0 && whole_codes(c, wide);
  DequantizeArgs a{};
  a.cache = view(c, first_layer);
  a.k = view(k);
  a.v = view(v);
  a.k_layer = k_layer_stride;
  a.v_layer = v_layer_stride;
  a.first = first_dev;
  a.count = count_dev;
  a.tokens = tokens;
  a.head_dim = c.head_dim;
  const int e = vector ? wide : 4;
  a.head_units = (c.head_dim + e - 1) / e;
  a.units = a.head_units * c.heads;
  a.by_head = Divide::by(a.head_units);
  a.span = std::min(a.units, kQuantThreads);
  a.by_span = Divide::by(a.span);
  a.tokens_at_once = kQuantThreads / a.span;
  // as many tokens to a workgroup as leave eight workgroups to a compute unit, kReadAtOnce units to a thread at most: 24 contexts of up to 8001 tokens take 294 us (a call in a loop 306), with 16 units
  // 4 % more, with 32 the same as with 16
  const int64_t all = (int64_t)tokens * a.units * batch * 2 * n_layers;
  const int per = std::max(1, (int)std::min<int64_t>(kReadAtOnce, all / (kQuantThreads * 2048)));
  a.at_a_time = std::max(1, std::min(kQuantTokens, per * kQuantThreads / a.units));
  const dim3 grid((tokens + a.at_a_time - 1) / a.at_a_time, 2 * n_layers, batch);
  choose(c.format, dtype, [&](auto form, auto type) {
    if (vector)
      hipLaunchKernelGGL((quantized_read_kernel<decltype(form)::value, decltype(type), true>), grid, dim3(kQuantThreads), 0, (hipStream_t)stream, a);
    else
      hipLaunchKernelGGL((quantized_read_kernel<decltype(form)::value, decltype(type), false>), grid, dim3(kQuantThreads), 0, (hipStream_t)stream, a);
  });
  return launched(who);
}

int dpllm_quantized_attention_workspace_bytes(int batch, int nodes, int heads, int kv_heads, int head_dim, int max_len, size_t* bytes) {
  const char* who = "dpllm_quantized_attention_workspace_bytes";
  if (!bytes) return refuse(DPLLM_EINVAL, "%s: bytes is NULL", who);
  if (int rc = check_attention(who, batch, nodes, heads, kv_heads, head_dim)) return rc;
  if (max_len < 0) return refuse(DPLLM_ESHAPE, "%s: max_len %d", who, max_len);
  *bytes = batch == 0 || nodes == 0 ? 0 : plan_quantized(batch, nodes, heads, kv_heads, head_dim, max_len).bytes;
  return DPLLM_OK;
}

int dpllm_quantized_attention(const dpllm_quantized_cache* cache, int layer, int batch, int nodes, int heads, int dtype, const int32_t* lens_dev, int max_len,
                              const dpllm_heads* q, const dpllm_heads* k_new, const dpllm_heads* v_new, const uint64_t* mask_dev, int64_t mask_stride, float scale,
                              const dpllm_heads* out, float* lse_dev, void* ws_dev, size_t ws_bytes, void* stream) {
  const char* who = "dpllm_quantized_attention";
  if (int rc = check_quantized(who, cache, batch)) return rc;
  if (dtype != DPLLM_F16 && dtype != DPLLM_BF16) return refuse(DPLLM_EINVAL, "%s: takes float16 and bfloat16, not dtype %d", who, dtype);
  if (int rc = check_attention(who, batch, nodes, heads, cache->heads, cache->head_dim)) return rc;
  if (layer < 0 || layer >= cache->layers) return refuse(DPLLM_ERANGE, "%s: layer %d of %d", who, layer, cache->layers);
  if (max_len < 0) return refuse(DPLLM_ESHAPE, "%s: max_len %d", who, max_len);
  if ((int64_t)cache->pages_per_seq * cache->page > INT32_MAX - 256) return refuse(DPLLM_ESHAPE, "%s: more than 2^31 - 256 tokens to a sequence", who);
  if (!std::isfinite(scale)) return refuse(DPLLM_EINVAL, "%s: scale is not finite", who);
  if (batch == 0 || nodes == 0) return DPLLM_OK;
  if (!lens_dev || !q || !out || !q->data || !out->data || !k_new != !v_new || (k_new && (!k_new->data || !v_new->data)))
    return refuse(DPLLM_EINVAL, "%s: a pointer is NULL (k_new and v_new may be, together)", who);
  const dpllm_quantized_cache c = reached(*cache);
  const dpllm_heads queries = reached(*q, batch, nodes, heads), results = reached(*out, batch, nodes, heads);
  const dpllm_heads keys = k_new ? reached(*k_new, batch, nodes, c.heads) : dpllm_heads{}, values = k_new ? reached(*v_new, batch, nodes, c.heads) : dpllm_heads{};
  if (!pieces(queries, 2) || !pieces(results, 2) || !pieces(keys, 2) || !pieces(values, 2) || ((uintptr_t)c.k | (uintptr_t)c.v) % 16 ||
      (c.layer_stride | c.page_stride | c.token_stride | c.head_stride) % 16)
    return refuse(DPLLM_EINVAL, "%s: tensors and codes have to be aligned to 16 bytes, with strides of whole 16 bytes", who);
  const QuantizedPlan p = plan_quantized(batch, nodes, heads, c.heads, c.head_dim, std::min<int64_t>(max_len, (int64_t)c.pages_per_seq * c.page));
  if (p.groups > 0x7fffff || (int64_t)batch * heads * nodes > 0x7fffff) return refuse(DPLLM_ESHAPE, "%s: %lld workgroups", who, (long long)p.groups);
  if (p.bytes > 0 && (!ws_dev || ws_bytes < p.bytes || (uintptr_t)ws_dev % 16))
    return refuse(DPLLM_ESTATE, "%s: needs a workspace of %zu bytes, aligned to 16", who, p.bytes);
  const QuantizedView w = view(c, layer);
  QuantizedArgs a{};
  a.cache = {w.k, w.v, 0, w.page_stride, w.token, w.head, w.table, w.table_stride, w.by_page, w.pages, w.page, w.pages_per_seq};
  a.k_scales = w.k_scales;
  a.v_scales = w.v_scales;
  a.scale_page = w.scale_page;
  a.scale_token = w.scale_token;
  a.scale_head = w.scale_head;
  fill_attention(a, p, batch, nodes, heads, c.heads, k_new != nullptr, scale);
  a.least = p.least;
  a.heads_at_once = p.heads;
  a.turns = p.turns;
  a.q = view(queries);
  a.out = view(results);
  a.k_new = view(keys);
  a.v_new = view(values);
  a.lens = lens_dev;
  a.mask = mask_dev;
  a.mask_stride = mask_stride;
  a.lse = lse_dev;
  place_workspace(a, p, ws_dev);
  if (c.format == DPLLM_CACHE_E4M3) launch_quantized<kE4m3>(dtype, c.head_dim, a, p, (hipStream_t)stream);
  if (c.format == DPLLM_CACHE_INT8) launch_quantized<kInt8>(dtype, c.head_dim, a, p, (hipStream_t)stream);
  if (c.format == DPLLM_CACHE_INT4) launch_quantized<kInt4>(dtype, c.head_dim, a, p, (hipStream_t)stream);
  return launched(who);
}

}  // extern "C"
