// Launches of the attention over a quantised cache; each format is compiled by itself.
#pragma once
#include "attention_plan.hpp"
#include "quantized_attention.hpp"

namespace dpllm {

// The split over a quantised cache.
struct QuantizedPlan : AttentionPlan {
  int heads, turns;      // of the kernel for few rows: kv heads that share a workgroup, and wavefronts to each
  int least;             // steps of the smallest part worth a workgroup
};

inline QuantizedPlan plan_quantized(int batch, int nodes, int heads, int kv_heads, int head_dim, int64_t max_len) {
  QuantizedPlan p{};
  p.rows = nodes * (heads / kv_heads);
  // Up to 64 rows go to wavefronts that take every step of codes apart by themselves, two tiles of rows at most to each, more to the kernel that shares that.  us with the former / with the latter, 4 sequences of
  // 9000 to 65001 tokens, heads of 128 (of 64): 36 to 64 rows, for which half the wavefronts of the latter have no rows, e4m3 106 / 134 (64 / 96), int8 112 / 139 (69 / 98), int4 93 / 144 (76 / 118); 100 rows e4m3
  // 175 / 148 (97 / 104), int8 187 / 149 (110 / 107), int4 156 / 156 (126 / 122).  (68 rows of int4 are past where they should be, 129 / 149; 240 rows over two sequences 134 to 154 / 126 to 133.)
  p.waves = p.rows <= 64 || head_dim == 256 ? 0 : p.rows <= 128 ? 4 : 8;
  p.mt = head_dim == 256 || p.rows <= 16 ? 1 : 2;
  p.tile = 16 * p.mt * std::max(p.waves, 1);
  p.row_tiles = (p.rows + p.tile - 1) / p.tile;
  const int64_t steps = (max_len + kAttTile - 1) / kAttTile + (nodes + kAttTile - 1) / kAttTile;
  p.lone = p.waves == 0 && p.mt == 1 && (head_dim == 64 || head_dim == 128) && steps <= 14;
  p.heads = p.lone || p.waves > 0 ? 1 : kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1;
  p.turns = (p.lone ? 8 : kAttWaves) / p.heads;
  p.least = p.waves > 0 ? kAttWaves : p.turns;
  const int64_t tiles = (int64_t)kv_heads / p.heads * p.row_tiles;
  const int64_t most = batch * ((steps + p.least - 1) / p.least), fill = ((p.waves == 8 ? 256 : 512) + tiles - 1) / tiles;
  p.slots = p.lone ? batch : (int)std::max<int64_t>(batch, std::min(most, fill >= 2 * batch ? fill : 3 * (int64_t)batch));
  p.groups = p.slots * tiles;
  const size_t part_rows = p.slots == batch ? 0 : (size_t)p.slots * kv_heads * p.row_tiles * p.tile;
  p.part = part_rows * head_dim * sizeof(float);
  p.stats = part_rows * sizeof(float2);
  p.bytes = part_rows == 0 ? 0 : p.part + p.stats + (size_t)batch * sizeof(int2);
  return p;
}

template <int FORMAT>
void launch_quantized(int dtype, int head_dim, const QuantizedArgs& a, const QuantizedPlan& p, hipStream_t s);

namespace {

template <int FORMAT, typename T, int D>
void launch_kernel(const QuantizedArgs& a, const QuantizedPlan& p, hipStream_t s) {
  const dim3 groups((unsigned)p.groups);
  if constexpr (D == 64 || D == 128)
    if (p.lone) hipLaunchKernelGGL((quantized_attention_kernel<FORMAT, T, D, 1, 8>), groups, dim3(8 * 64), 0, s, a);
  if constexpr (D < 256) {
    if (p.waves == 4) hipLaunchKernelGGL((quantized_attention_wide_kernel<FORMAT, T, D, 2, 4>), groups, dim3(4 * 64), 0, s, a);
    if (p.waves == 8) hipLaunchKernelGGL((quantized_attention_wide_kernel<FORMAT, T, D, 2, 8>), groups, dim3(8 * 64), 0, s, a);
  }
  if (p.waves == 0 && p.mt == 1 && !p.lone) hipLaunchKernelGGL((quantized_attention_kernel<FORMAT, T, D, 1, kAttWaves>), groups, dim3(kAttWaves * 64), 0, s, a);
  if constexpr (D < 256)
    if (p.waves == 0 && p.mt == 2) hipLaunchKernelGGL((quantized_attention_kernel<FORMAT, T, D, 2, kAttWaves>), groups, dim3(kAttWaves * 64), 0, s, a);
  if (p.bytes > 0) {
    const dim3 rows((uint32_t)a.batch * a.kv_heads * a.rows);
    const Divide by_rows = Divide::by(a.rows), by_heads = Divide::by(a.kv_heads), by_tile = Divide::by(p.tile);
    if (p.slots >= 32 * a.batch)
      hipLaunchKernelGGL((quantized_join_kernel<T, D, 512>), rows, dim3(512), 0, s, a, p.tile, by_rows, by_heads, by_tile);
    else
      hipLaunchKernelGGL((quantized_join_kernel<T, D, 128>), rows, dim3(128), 0, s, a, p.tile, by_rows, by_heads, by_tile);
  }
}

template <int FORMAT, typename T>
void launch_head_dim(int head_dim, const QuantizedArgs& a, const QuantizedPlan& p, hipStream_t s) {
  if (head_dim == 64) launch_kernel<FORMAT, T, 64>(a, p, s);
  if (head_dim == 96) launch_kernel<FORMAT, T, 96>(a, p, s);
  if (head_dim == 128) launch_kernel<FORMAT, T, 128>(a, p, s);
  if (head_dim == 256) launch_kernel<FORMAT, T, 256>(a, p, s);
}

template <int FORMAT>
void launch_dtype(int dtype, int head_dim, const QuantizedArgs& a, const QuantizedPlan& p, hipStream_t s) {
  if (dtype == DPLLM_F16)
    launch_head_dim<FORMAT, half_t>(head_dim, a, p, s);
  else
    launch_head_dim<FORMAT, bfloat_t>(head_dim, a, p, s);
}

}  // namespace
}  // namespace dpllm
