// Launches of the attention over a quantised cache; each format is compiled by itself.
#pragma once
#include "attention_plan.hpp"
#include "quantized_attention.hpp"

namespace dpllm {

template <int FORMAT>
void launch_quantized(int dtype, int head_dim, const QuantizedArgs& a, const AttentionPlan& p, hipStream_t s);

namespace {

template <int FORMAT, typename T, int D>
void launch_kernel(const QuantizedArgs& a, const AttentionPlan& p, hipStream_t s) {
  const dim3 groups((unsigned)p.groups);
  if constexpr (D == 64 || D == 128)
    if (p.lone) hipLaunchKernelGGL((quantized_attention_kernel<FORMAT, T, D, 1, 8>), groups, dim3(8 * 64), 0, s, a);
  if (p.waves == 0 && p.mt == 1 && !p.lone) hipLaunchKernelGGL((quantized_attention_kernel<FORMAT, T, D, 1, kAttWaves>), groups, dim3(kAttWaves * 64), 0, s, a);
  if constexpr (D < 256)
    if (p.waves == 0 && p.mt == 2) hipLaunchKernelGGL((quantized_attention_kernel<FORMAT, T, D, 2, kAttWaves>), groups, dim3(kAttWaves * 64), 0, s, a);
  if (p.bytes > 0) {
    const uint32_t all_rows = (uint32_t)a.batch * a.kv_heads * a.rows;
    hipLaunchKernelGGL((tree_attention_join_kernel<T, D>), dim3((all_rows + 3) / 4), dim3(256), 0, s, a, p.tile, Divide::by(a.rows), Divide::by(a.kv_heads),
                       Divide::by(p.tile), all_rows);
  }
}

template <int FORMAT, typename T>
void launch_head_dim(int head_dim, const QuantizedArgs& a, const AttentionPlan& p, hipStream_t s) {
  if (head_dim == 64) launch_kernel<FORMAT, T, 64>(a, p, s);
  if (head_dim == 96) launch_kernel<FORMAT, T, 96>(a, p, s);
  if (head_dim == 128) launch_kernel<FORMAT, T, 128>(a, p, s);
  if (head_dim == 256) launch_kernel<FORMAT, T, 256>(a, p, s);
}

template <int FORMAT>
void launch_dtype(int dtype, int head_dim, const QuantizedArgs& a, const AttentionPlan& p, hipStream_t s) {
  if (dtype == DPLLM_F16)
    launch_head_dim<FORMAT, half_t>(head_dim, a, p, s);
  else
    launch_head_dim<FORMAT, bfloat_t>(head_dim, a, p, s);
}

}  // namespace
}  // namespace dpllm
