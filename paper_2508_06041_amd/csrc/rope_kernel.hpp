// Rotary positions.  The pair (a, b) of a token at position pos becomes s (a cos t - b sin t, a sin t + b cos t), t = pos * f of the pair;
// the transpose, which the gradient needs, is the same with -t.  Elements past the rotated part are copied.
#pragma once
#include "token_common.hpp"

namespace dpllm {

constexpr int kRopeTensors = 4;
constexpr int kRopeThreads = 256;

struct RopeArgs {
  Heads x[kRopeTensors], out[kRopeTensors];
  int end[kRopeTensors];        // heads of the tensors up to and with this one
  const double* freqs;          // radians per position, one per pair
  const int32_t* positions;     // [batch][tokens]
  int64_t positions_stride;     // per sequence; 0: the same for all
  Divide by_tokens, by_units, by_row, by_pairs;
  int64_t all;                  // batch * tokens
  int tokens, heads, pairs, rotary, units, turned, at_a_time;
  float scale;
  int inverse;
};

// Angles are formed in 64 bits as turns of which the whole ones are dropped: a position of 2^20 has used up 20 of the 24 bits of a float,
// in 64 bits the angle of a position below 2^31 is off by less than 1e-6.  What is left, at most half a turn, goes on in 32 bits.
// A workgroup forms the sines of its tokens once, in LDS, for all heads of all tensors (queries and keys in one launch).
// E: elements a thread moves at a time, 16 bytes; 1 where the layout does not allow that.
template <typename T, int E, bool HALF>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeArgs a) {
  extern __shared__ float2 turn[];   // [at_a_time][pairs]
  typedef T vec __attribute__((ext_vector_type(E)));
  for (int64_t first = (int64_t)blockIdx.x * a.at_a_time; first < a.all; first += (int64_t)gridDim.x * a.at_a_time) {
  const int n = (int)(a.all - first < a.at_a_time ? a.all - first : a.at_a_time);
  for (uint32_t i = threadIdx.x; i < (uint32_t)(n * a.pairs); i += kRopeThreads) {
    const uint32_t tok = a.by_pairs.of(i), p = i - tok * a.pairs;
    const uint32_t at = (uint32_t)(first + tok), b = a.by_tokens.of(at);
    const double angle = (double)a.positions[b * a.positions_stride + (at - b * a.tokens)] * a.freqs[p];
    double t = angle * 0.15915494309189533577;   // 1 / (2 pi)
    t -= __builtin_rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    turn[i] = make_float2(c * a.scale, (a.inverse ? -s : s) * a.scale);
  }
  __syncthreads();
  const uint32_t row_units = (uint32_t)a.heads * a.units;
  for (uint32_t i = threadIdx.x; i < n * row_units; i += kRopeThreads) {
    const uint32_t tok = a.by_row.of(i), in_row = i - tok * row_units;
    uint32_t head = a.by_units.of(in_row);
    const uint32_t unit = in_row - head * a.units;
    int w = 0;
    while (head >= (uint32_t)a.end[w]) ++w;
    if (w > 0) head -= a.end[w - 1];
    const uint32_t at = (uint32_t)(first + tok), b = a.by_tokens.of(at), t = at - b * a.tokens;
    const Heads &x = a.x[w], &o = a.out[w];
    const T* src = reinterpret_cast<const T*>(x.data) + b * x.batch_stride + t * x.token_stride + head * x.head_stride;
    T* dst = reinterpret_cast<T*>(o.data) + b * o.batch_stride + t * o.token_stride + head * o.head_stride;
    if (unit >= (uint32_t)a.turned) {
      const int d = a.rotary + (unit - a.turned) * E;
      *reinterpret_cast<vec*>(dst + d) = *reinterpret_cast<const vec*>(src + d);
      continue;
    }
    const float2* cs = turn + tok * a.pairs;
    if constexpr (HALF) {
      const int d = unit * E;
      const vec va = *reinterpret_cast<const vec*>(src + d), vb = *reinterpret_cast<const vec*>(src + a.pairs + d);
      vec ra, rb;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 f = cs[d + e];
        const float p = (float)va[e], q = (float)vb[e];
        ra[e] = (T)(p * f.x - q * f.y);
        rb[e] = (T)(p * f.y + q * f.x);
      }
      *reinterpret_cast<vec*>(dst + d) = ra;
      *reinterpret_cast<vec*>(dst + a.pairs + d) = rb;
    } else {
      constexpr int P = E > 1 ? E / 2 : 1;   // pairs of a unit
      typedef T two __attribute__((ext_vector_type(2 * P)));
      const int d = unit * 2 * P;
      two v;
      if constexpr (E > 1) {
        v = *reinterpret_cast<const two*>(src + d);
      } else {
        v[0] = src[d];
        v[1] = src[d + 1];
      }
#pragma unroll
      for (int e = 0; e < P; ++e) {
        const float2 f = cs[unit * P + e];
        const float p = (float)v[2 * e], q = (float)v[2 * e + 1];
        v[2 * e] = (T)(p * f.x - q * f.y);
        v[2 * e + 1] = (T)(p * f.y + q * f.x);
      }
      if constexpr (E > 1) {
        *reinterpret_cast<two*>(dst + d) = v;
      } else {
        dst[d] = v[0];
        dst[d + 1] = v[1];
      }
    }
  }
  __syncthreads();   // the next tokens' sines take the place of these
  }
}

}  // namespace dpllm
