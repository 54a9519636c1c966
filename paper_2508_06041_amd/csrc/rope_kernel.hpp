// Rotary positions.  The pair (a, b) of a token at position pos becomes s (a cos t - b sin t, a sin t + b cos t), t = pos * f of the pair;
// the transpose, which the gradient needs, is the same with -t.  Elements past the rotated part are copied.
#pragma once
#include "token_common.hpp"

namespace dpllm {

constexpr int kRopeTensors = 4;
constexpr int kRopeThreads = 256;
constexpr int kRopeAtOnce = 2;      // units that a thread has on their way (537 MB of gradient: 1 and 2 98 us, 4 109)

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

// What a thread moves at a time: 16 bytes (or an element, E = 1, where the layout does not allow that) and, of a head whose pairs lie half the rotated
// part apart, the 16 bytes that go with them.
template <typename T, int E>
struct RopeUnit {
  typedef T vec __attribute__((ext_vector_type(E)));
  vec a, b;
  char* to;
  uint32_t tok, unit;
  bool turns;
};

// Angles are formed in 64 bits as turns of which the whole ones are dropped: a position of 2^20 has used up 20 of the 24 bits of a float,
// in 64 bits the angle of a position below 2^31 is off by less than 1e-6.  What is left, at most half a turn, goes on in 32 bits.
// A workgroup forms the sines of its tokens once, in LDS, for all heads of all tensors (queries and keys in one launch); its first units are on
// their way meanwhile.
// Bound by memory: 537 MB of gradient in 98 us, 5.5 TB/s (a plain copy of 2 GiB: 4.6); a launch of one token takes 3 us of latency.
template <typename T, int E, bool HALF>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeArgs a) {
  extern __shared__ float2 turn[];   // [at_a_time][pairs]
  typedef RopeUnit<T, E> Unit;
  typedef typename Unit::vec vec;
  constexpr int P = HALF ? E : E > 1 ? E / 2 : 1;      // pairs of a unit
  const uint32_t row_units = (uint32_t)a.heads * a.units;
  for (int64_t first = (int64_t)blockIdx.x * a.at_a_time; first < a.all; first += (int64_t)gridDim.x * a.at_a_time) {
    const uint32_t n = (uint32_t)(a.all - first < a.at_a_time ? a.all - first : a.at_a_time), end = n * row_units;
    Unit u[kRopeAtOnce];
    auto load = [&](uint32_t i, Unit& x) {
      if (i >= end) return;
      x.tok = a.by_row.of(i);
      const uint32_t in_row = i - x.tok * row_units;
      uint32_t head = a.by_units.of(in_row);
      x.unit = in_row - head * a.units;
      int w = 0;
      while (head >= (uint32_t)a.end[w]) ++w;
      if (w > 0) head -= a.end[w - 1];
      const uint32_t at = (uint32_t)(first + x.tok), b = a.by_tokens.of(at), t = at - b * a.tokens;
      const Heads &from = a.x[w], &to = a.out[w];
      x.turns = x.unit < (uint32_t)a.turned;
      const uint32_t d = x.turns ? x.unit * (HALF ? E : 2 * P) : a.rotary + (x.unit - a.turned) * E;
      const T* src = reinterpret_cast<const T*>(from.data) + b * from.batch_stride + t * from.token_stride + head * from.head_stride + d;
      x.to = to.data + (b * to.batch_stride + t * to.token_stride + head * to.head_stride + d) * (int64_t)sizeof(T);
      x.a = *reinterpret_cast<const vec*>(src);
      if (x.turns && (HALF || E == 1)) x.b = *reinterpret_cast<const vec*>(src + (HALF ? a.pairs : 1));
    };
    auto store = [&](uint32_t i, Unit& x) {
      if (i >= end) return;
      T* to = reinterpret_cast<T*>(x.to);
      if (x.turns) {
        const float2* cs = turn + x.tok * a.pairs + x.unit * P;
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float2 f = cs[e];
          constexpr bool apart = HALF || E == 1;
          const float p = (float)(apart ? x.a[e] : x.a[2 * e % E]), q = (float)(apart ? x.b[e % E] : x.a[(2 * e + 1) % E]);
          const T r = (T)(p * f.x - q * f.y), s = (T)(p * f.y + q * f.x);
          if constexpr (apart) {
            x.a[e] = r;
            x.b[e] = s;
          } else {
            x.a[2 * e % E] = r;
            x.a[(2 * e + 1) % E] = s;
          }
        }
        if constexpr (HALF || E == 1) *reinterpret_cast<vec*>(to + (HALF ? a.pairs : 1)) = x.b;
      }
      *reinterpret_cast<vec*>(to) = x.a;
    };
#pragma unroll
    for (int k = 0; k < kRopeAtOnce; ++k) load(threadIdx.x + k * kRopeThreads, u[k]);
    for (uint32_t i = threadIdx.x; i < n * a.pairs; i += kRopeThreads) {
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
    for (uint32_t i = threadIdx.x; i < end; i += kRopeAtOnce * kRopeThreads) {
      if (i != threadIdx.x)
#pragma unroll
        for (int k = 0; k < kRopeAtOnce; ++k) load(i + k * kRopeThreads, u[k]);
#pragma unroll
      for (int k = 0; k < kRopeAtOnce; ++k) store(i + k * kRopeThreads, u[k]);
    }
    __syncthreads();   // the next tokens' sines take the place of these
  }
}

}  // namespace dpllm
