// Exchanges between the lanes of a wavefront.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace dpllm {

// The value of another lane: STEP 0 and 1 exchange inside four lanes, 2 and 3 the fours of eight and the eights of sixteen, 4 and 5 sixteens and halves.  With all six
// every lane has met every other, without LDS; two lanes that meet form the same sum, so all end with the same bits.
template <int STEP>
__device__ __forceinline__ uint32_t other(uint32_t v) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  if constexpr (STEP < 4) {
    constexpr int control = STEP == 0 ? 0xb1 : STEP == 1 ? 0x4e : STEP == 2 ? 0x141 : 0x140;
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, control, 0xf, 0xf, true);
  } else {
    const u32x2 p = STEP == 4 ? __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(v, v, false, false))
                              : __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(v, v, false, false));
    const uint32_t first = p[0], second = p[1];      // of a pair of rows (halves), in both
    const bool upper = (threadIdx.x >> STEP) & 1;
    return upper ? first : second;
  }
}
template <int STEP>
__device__ __forceinline__ float other(float v) { return __uint_as_float(other<STEP>(__float_as_uint(v))); }
template <int STEP>
__device__ __forceinline__ int other(int v) { return (int)other<STEP>((uint32_t)v); }
template <int STEP>
__device__ __forceinline__ double other(double v) {
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)other<STEP>((uint32_t)(w >> 32)) << 32 | other<STEP>((uint32_t)w));
}
template <typename T, typename F>
__device__ __forceinline__ T wave_all(T v, F f) {
  v = f(v, other<0>(v));
  v = f(v, other<1>(v));
  v = f(v, other<2>(v));
  v = f(v, other<3>(v));
  v = f(v, other<4>(v));
  return f(v, other<5>(v));
}
__device__ __forceinline__ double wave_sum(double v) {
  return wave_all(v, [](double a, double b) { return a + b; });
}

// The same over groups of L = 1, 2, ... 64 neighbouring lanes (the same L for all): every lane of a group has its group's answer.
template <typename T, typename F>
__device__ __forceinline__ T team_all(T v, int lanes, F f) {
  if (lanes > 1) v = f(v, other<0>(v));
  if (lanes > 2) v = f(v, other<1>(v));
  if (lanes > 4) v = f(v, other<2>(v));
  if (lanes > 8) v = f(v, other<3>(v));
  if (lanes > 16) v = f(v, other<4>(v));
  if (lanes > 32) v = f(v, other<5>(v));
  return v;
}

}  // namespace dpllm
