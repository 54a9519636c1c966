// How the attention calls split their work, and what sizes they take.
#pragma once
#include <algorithm>
#include <cmath>

#include "token_host.hpp"
#include "tree_attention.hpp"

namespace dpllm {

// Which kernel, and how the work is split.
struct AttentionPlan {
  int rows, mt, waves;   // rows of a kv head; tiles of 16 rows to a wavefront; waves > 0: the kernel for many rows with so many wavefronts
  int tile, row_tiles, slots;
  bool lone;             // the kernel for few rows with twice the wavefronts, one workgroup to a sequence and kv head
  int64_t groups;        // workgroups
  size_t part, stats, bytes;
};

inline AttentionPlan plan_attention(int batch, int nodes, int heads, int kv_heads, int head_dim, int64_t max_len) {
  AttentionPlan p;
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

inline void place_workspace(AttentionArgs& a, const AttentionPlan& p, void* ws) {
  if (p.bytes == 0) return;
  a.part = (float*)ws;
  a.stats = (float2*)((char*)ws + p.part);
  a.places = (int2*)((char*)ws + p.part + p.stats);
}

// The sizes and the scale.
inline void fill_attention(AttentionArgs& a, const AttentionPlan& p, int batch, int nodes, int heads, int kv_heads, bool sees_nodes, float scale) {
  a.scale = std::fabs(scale);
  a.scale_log2 = (float)(std::fabs((double)scale) * 1.44269504088896340736);
  a.sign = scale < 0 ? 0x80008000u : 0u;
  a.keep = scale == 0 ? 0u : ~0u;
  if (scale == 0) a.scale_log2 = 1.f;      // scores of 0, and a scale that the tops can be measured with
  a.group = heads / kv_heads;
  a.by_group = Divide::by(a.group);
  a.nodes = nodes;
  a.seen_nodes = sees_nodes ? nodes : 0;
  a.words = (nodes + 63) / 64;
  a.kv_heads = kv_heads;
  a.rows = p.rows;
  a.row_tiles = p.row_tiles;
  a.batch = batch;
  a.slots = p.slots;
  a.least = kAttWaves;
}

inline int check_attention(const char* who, int batch, int nodes, int heads, int kv_heads, int head_dim) {
  if (batch < 0 || batch > 65536 || nodes < 0 || nodes > DPLLM_MAX_NODES)
    return refuse(DPLLM_ESHAPE, "%s: %d sequences of %d nodes (at most 65536 of %d)", who, batch, nodes, DPLLM_MAX_NODES);
  if (heads < 1 || heads > 1024 || kv_heads < 1 || heads % kv_heads) return refuse(DPLLM_ESHAPE, "%s: %d heads over %d", who, heads, kv_heads);
  if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 256) return refuse(DPLLM_ESHAPE, "%s: head_dim %d (64, 96, 128 or 256)", who, head_dim);
  return DPLLM_OK;
}

}  // namespace dpllm
