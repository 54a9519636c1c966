// The attention over a cache of int4 codes; see quantized_attention.hpp.
#include <hip/hip_runtime.h>

#include "quantized_launch.hpp"

namespace dpllm {
template <>
void launch_quantized<kInt4>(int dtype, int head_dim, const QuantizedArgs& a, const QuantizedPlan& p, hipStream_t s) {
  launch_dtype<kInt4>(dtype, head_dim, a, p, s);
}
}  // namespace dpllm
