// Host side of dpllm_tree_attention: argument checks, how the work is split, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "token_host.hpp"
#include "tree_attention.hpp"

using namespace dpllm;

namespace {

// Which kernel, and how the work is split.
struct Plan {
  int rows, mt, waves;   // rows of a kv head; tiles of 16 rows to a wavefront; waves > 0: the kernel for many rows with so many wavefronts
  int tile, row_tiles, slots;
  bool lone;             // the kernel for few rows with twice the wavefronts, one workgroup to a sequence and kv head
  int64_t groups;        // workgroups
  size_t part, stats, bytes;
};

Plan plan_of(int batch, int nodes, int heads, int kv_heads, int head_dim, int64_t max_len) {
  Plan p;
  p.rows = nodes * (heads / kv_heads);
  p.waves = p.rows <= 32 ? 0 : p.rows <= 128 || head_dim == 256 ? 4 : 8;
  p.mt = head_dim == 256 || p.rows <= 16 || (p.rows > 32 && p.rows <= 64) ? 1 : 2;
  p.tile = 16 * p.mt * std::max(p.waves, 1);
  p.row_tiles = (p.rows + p.tile - 1) / p.tile;
  // Workgroups: as many as run at once, two to a compute unit (one of eight wavefronts); more parts are more results to write and join (63 nodes over
  // 130001 tokens 179 us with 256 workgroups, 213 with 512, 242 with 1024; four sequences of 8 nodes 43.6 with 512, 45.9 with 1024).  With many
  // sequences three parts each, so that long ones do not hold up the rest.
  const int64_t steps = (max_len + kAttTile - 1) / kAttTile + (nodes + kAttTile - 1) / kAttTile, tiles = (int64_t)kv_heads * p.row_tiles;
  const int64_t most = batch * ((steps + kAttWaves - 1) / kAttWaves), fill = ((p.waves == 8 ? 256 : 512) + tiles - 1) / tiles;
  // short contexts: eight wavefronts take them in two turns, which is faster than four and a second launch to join the parts (one token of 32 heads
  // over 8, us in a graph, over 200 tokens 7.3 against 9.1, over 500 9.5 against 8.9)
  p.lone = p.waves == 0 && p.mt == 1 && (head_dim == 64 || head_dim == 128) && steps <= 14;
  p.slots = p.lone ? batch : (int)std::max<int64_t>(batch, std::min(most, fill >= 2 * batch ? fill : 3 * (int64_t)batch));
  p.groups = p.slots * tiles;
  const bool whole = p.slots == batch;
  p.part = whole ? 0 : (size_t)p.groups * p.tile * head_dim * sizeof(float);
  p.stats = whole ? 0 : (size_t)p.groups * p.tile * sizeof(float2);
  p.bytes = whole ? 0 : p.part + p.stats + (size_t)batch * sizeof(int2);
  return p;
}

template <typename T, int D>
void launch(const AttentionArgs& a, const Plan& p, hipStream_t s) {
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
void launch(int head_dim, const AttentionArgs& a, const Plan& p, hipStream_t s) {
  if (head_dim == 64) launch<T, 64>(a, p, s);
  if (head_dim == 96) launch<T, 96>(a, p, s);
  if (head_dim == 128) launch<T, 128>(a, p, s);
  if (head_dim == 256) launch<T, 256>(a, p, s);
}

int check_sizes(const char* who, int batch, int nodes, int heads, int kv_heads, int head_dim) {
  if (batch < 0 || batch > 65536 || nodes < 0 || nodes > DPLLM_MAX_NODES)
    return refuse(DPLLM_ESHAPE, "%s: %d sequences of %d nodes (at most 65536 of %d)", who, batch, nodes, DPLLM_MAX_NODES);
  if (heads < 1 || heads > 1024 || kv_heads < 1 || heads % kv_heads) return refuse(DPLLM_ESHAPE, "%s: %d heads over %d", who, heads, kv_heads);
  if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 256) return refuse(DPLLM_ESHAPE, "%s: head_dim %d (64, 96, 128 or 256)", who, head_dim);
  return DPLLM_OK;
}

}  // namespace

extern "C" {

int dpllm_tree_attention_workspace_bytes(int batch, int nodes, int heads, int kv_heads, int head_dim, int max_len, size_t* bytes) {
  const char* who = "dpllm_tree_attention_workspace_bytes";
  if (!bytes) return refuse(DPLLM_EINVAL, "%s: bytes is NULL", who);
  if (int rc = check_sizes(who, batch, nodes, heads, kv_heads, head_dim)) return rc;
  if (max_len < 0) return refuse(DPLLM_ESHAPE, "%s: max_len %d", who, max_len);
  *bytes = batch == 0 || nodes == 0 ? 0 : plan_of(batch, nodes, heads, kv_heads, head_dim, max_len).bytes;
  return DPLLM_OK;
}

int dpllm_tree_attention(const dpllm_cache* cache, int layer, int batch, int nodes, int heads, const int32_t* lens_dev, int max_len,
                         const dpllm_heads* q, const dpllm_heads* k_new, const dpllm_heads* v_new, const uint64_t* mask_dev, int64_t mask_stride,
                         float scale, const dpllm_heads* out, float* lse_dev, void* ws_dev, size_t ws_bytes, void* stream) {
  const char* who = "dpllm_tree_attention";
  if (int rc = check_cache(who, cache, batch)) return rc;
  if (cache->dtype == DPLLM_F32) return refuse(DPLLM_EINVAL, "%s: takes float16 and bfloat16", who);
  if (int rc = check_sizes(who, batch, nodes, heads, cache->heads, cache->head_dim)) return rc;
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
  const Plan p = plan_of(batch, nodes, heads, cache->heads, cache->head_dim, std::min<int64_t>(max_len, (int64_t)cache->pages_per_seq * cache->page));
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
  if (p.bytes > 0) {
    a.part = (float*)ws_dev;
    a.stats = (float2*)((char*)ws_dev + p.part);
    a.places = (int2*)((char*)ws_dev + p.part + p.stats);
  }
  a.scale = std::fabs(scale);
  a.scale_log2 = (float)(std::fabs((double)scale) * 1.44269504088896340736);
  a.sign = scale < 0 ? 0x80008000u : 0u;
  a.keep = scale == 0 ? 0u : ~0u;
  if (scale == 0) a.scale_log2 = 1.f;      // scores of 0, and a scale that the tops can be measured with
  a.group = heads / cache->heads;
  a.by_group = Divide::by(a.group);
  a.nodes = nodes;
  a.seen_nodes = k_new ? nodes : 0;
  a.words = (nodes + 63) / 64;
  a.kv_heads = cache->heads;
  a.rows = p.rows;
  a.row_tiles = p.row_tiles;
  a.batch = batch;
  a.slots = p.slots;
  a.least = kAttWaves;
  if (cache->dtype == DPLLM_F16)
    launch<half_t>(cache->head_dim, a, p, (hipStream_t)stream);
  else
    launch<bfloat_t>(cache->head_dim, a, p, (hipStream_t)stream);
  return launched(who);
}

}  // extern "C"
