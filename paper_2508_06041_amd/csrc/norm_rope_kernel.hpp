// Norms of heads with learned weights and their rotary positions in one pass, and the gradient of that.
//   r = 1 / sqrt(mean(x^2) + eps), y = R (w r x), R the rotation of rope_kernel.hpp (or none)
//   with h = R^T g and S = sum of w h x over the head: dx = r w h - x r^3 S / head_dim, dw = the sum of h r x over tokens and heads that share w
#pragma once
#include "lanes.hpp"
#include "token_common.hpp"

namespace dpllm {

constexpr int kNormTensors = DPLLM_MAX_TENSORS;
constexpr int kNormThreads = 256;

struct NormArgs {
  Heads x[kNormTensors], g[kNormTensors], out[kNormTensors];      // g: gradients of the outputs
  const void* weights[kNormTensors];
  int64_t weight_strides[kNormTensors];
  int end[kNormTensors];        // heads of the tensors up to and with this one
  const double* freqs;          // radians per position, one per pair
  const int32_t* positions;     // [batch][tokens]
  int64_t positions_stride;     // per sequence; 0: the same for all
  Divide by_tokens, by_heads, by_pairs;
  int64_t all;                  // batch * tokens
  int tokens, heads, head_dim, pairs, rotary, units, turned, lanes, log_lanes, at_a_time, weight_dtype;
  float eps, scale;
};

// What a lane has of a head: E elements, or where the two of a pair lie apart (HALF: half the rotated part; E = 1: neighbours) E and those E that go with them.
// Units from `turned` on are not rotated and have only the first E.
template <typename T, int E, bool HALF>
struct NormUnit {
  static constexpr bool APART = HALF || E == 1;
  static constexpr int N = APART ? 2 * E : E;
  typedef T vec __attribute__((ext_vector_type(E)));
  float v[N];
  __device__ __forceinline__ static int place(const NormArgs& a, int u) { return u < a.turned ? u * (APART && !HALF ? 2 : E) : a.rotary + (u - a.turned) * E; }
  template <typename S>
  __device__ __forceinline__ void read(const NormArgs& a, const S* head, int u) {
    typedef S some __attribute__((ext_vector_type(E)));
    const S* p = head + place(a, u);
    const some x = *reinterpret_cast<const some*>(p);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (float)x[e];
    if constexpr (APART) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[E + e] = 0.f;
      if (u < a.turned) {
        const some y = *reinterpret_cast<const some*>(p + (HALF ? a.pairs : 1));
#pragma unroll
        for (int e = 0; e < E; ++e) v[E + e] = (float)y[e];
      }
    }
  }
  __device__ __forceinline__ void read_weight(const NormArgs& a, int tensor, int head, int u) {
    const void* w = a.weights[tensor];
    const int64_t at = head * a.weight_strides[tensor];
    if (w == nullptr) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = 1.f;
    } else if (a.weight_dtype == DPLLM_F32) {
      read(a, static_cast<const float*>(w) + at, u);
    } else if (a.weight_dtype == DPLLM_F16) {
      read(a, static_cast<const half_t*>(w) + at, u);
    } else {
      read(a, static_cast<const bfloat_t*>(w) + at, u);
    }
  }
  __device__ __forceinline__ void write(const NormArgs& a, T* head, int u) const {
    T* p = head + place(a, u);
    vec x;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = (T)v[e];
    if constexpr (APART) {
      if (u < a.turned) {
        vec y;
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = (T)v[E + e];
        *reinterpret_cast<vec*>(p + (HALF ? a.pairs : 1)) = y;
      }
    }
    *reinterpret_cast<vec*>(p) = x;
  }
  // Turned by the angles of its pairs, cs: cosine and sine times the scale; BACK: the transpose.
  template <bool BACK>
  __device__ __forceinline__ void turn(const NormArgs& a, const float2* cs, int u) {
    if (u >= a.turned) return;
    constexpr int P = HALF ? E : E > 1 ? E / 2 : 1;
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const float2 f = cs[u * P + e];
      const int i = APART ? e : 2 * e, j = APART ? E + e : 2 * e + 1;
      const float p = v[i], q = v[j], s = BACK ? -f.y : f.y;
      v[i] = p * f.x - q * s;
      v[j] = p * s + q * f.x;
    }
  }
};

__device__ __forceinline__ float plus(float a, float b) { return a + b; }

// The sines of n tokens from `first` on; a barrier has to follow.
__device__ __forceinline__ void fill_sines(const NormArgs& a, int64_t first, int n, float2* sines) {
  for (uint32_t i = threadIdx.x; i < (uint32_t)n * a.pairs; i += kNormThreads) {
    const uint32_t tok = a.by_pairs.of(i), p = i - tok * a.pairs, at = (uint32_t)(first + tok), b = a.by_tokens.of(at);
    const double angle = (double)a.positions[b * a.positions_stride + (at - b * a.tokens)] * a.freqs[p];
    double t = angle * 0.15915494309189533577;   // 1 / (2 pi); as in rope_kernel.hpp
    t -= __builtin_rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    sines[i] = make_float2(c * a.scale, s * a.scale);
  }
}

// One group of `lanes` lanes to a head.  ONE: a head has no more units than lanes, and is read once; else it is read again behind its sum.
template <typename T, int E, bool HALF, bool ONE>
__global__ void __launch_bounds__(kNormThreads) norm_rope_kernel(const NormArgs a) {
  extern __shared__ float2 sines[];   // [at_a_time][pairs]
  typedef NormUnit<T, E, HALF> Unit;
  const int lane = threadIdx.x & (a.lanes - 1), team = threadIdx.x >> a.log_lanes, teams = kNormThreads >> a.log_lanes;
  const float by = 1.0f / (float)a.head_dim;
  for (int64_t first = (int64_t)blockIdx.x * a.at_a_time; first < a.all; first += (int64_t)gridDim.x * a.at_a_time) {
    const int n = (int)(a.all - first < a.at_a_time ? a.all - first : a.at_a_time), rows = n * a.heads;
    struct Row {
      const T* from;
      T* to;
      int tok, tensor, head;
      Unit x;
    };
    auto find = [&](int i, Row& r) {
      r.tok = a.by_heads.of(i);
      r.head = i - r.tok * a.heads;
      r.tensor = 0;
      while (r.head >= a.end[r.tensor]) ++r.tensor;
      if (r.tensor > 0) r.head -= a.end[r.tensor - 1];
      const uint32_t at = (uint32_t)(first + r.tok), b = a.by_tokens.of(at), t = at - b * a.tokens;
      const Heads &from = a.x[r.tensor], &to = a.out[r.tensor];
      r.from = reinterpret_cast<const T*>(from.data) + b * from.batch_stride + t * from.token_stride + r.head * from.head_stride;
      r.to = reinterpret_cast<T*>(to.data) + b * to.batch_stride + t * to.token_stride + r.head * to.head_stride;
      if (ONE && lane < a.units) r.x.read(a, r.from, lane);
    };
    Row row;
    if (team < rows) find(team, row);
    fill_sines(a, first, n, sines);
    __syncthreads();
    for (int i = team; i < rows; i += teams) {
      Row next;
      if (i + teams < rows) find(i + teams, next);
      float sum = 0.f;
      for (int u = lane; u < a.units; u += a.lanes) {
        if (!ONE) row.x.read(a, row.from, u);
#pragma unroll
        for (int e = 0; e < Unit::N; ++e) sum = __builtin_fmaf(row.x.v[e], row.x.v[e], sum);
      }
      sum = team_all(sum, a.lanes, plus);
      const float r = 1.0f / __builtin_sqrtf(sum * by + a.eps);
      for (int u = lane; u < a.units; u += a.lanes) {
        if (!ONE) row.x.read(a, row.from, u);
        Unit w;
        w.read_weight(a, row.tensor, row.head, u);
#pragma unroll
        for (int e = 0; e < Unit::N; ++e) row.x.v[e] = row.x.v[e] * r * w.v[e];
        row.x.template turn<false>(a, sines + row.tok * a.pairs, u);
        row.x.write(a, row.to, u);
      }
      row = next;
    }
    __syncthreads();   // the next tokens' sines take the place of these
  }
}

struct NormBackArgs {
  NormArgs n;
  float* parts;                      // [workgroup][head_dim]
  int first[kNormTensors + 1];       // the first workgroup of a tensor
  int splits[kNormTensors];          // workgroups to a weight
  int group_heads[kNormTensors];     // heads that share one
  Divide by_group[kNormTensors], by_splits[kNormTensors];
  int64_t tokens_each[kNormTensors];      // tokens to a workgroup
  void* grad_weights[kNormTensors];
  int groups_end[kNormTensors];      // weights of the tensors up to and with this one
};

// A workgroup takes the heads that share one weight (all of a tensor's, or one) of a stretch of tokens, so that a lane has the same elements of the same weight throughout
// and adds their gradient up in registers (in LDS where it has several units); the groups of lanes meet in LDS at the end, in their order.
template <typename T, int E, bool HALF, bool ONE>
__global__ void __launch_bounds__(kNormThreads) norm_rope_backward_kernel(const NormBackArgs k) {
  extern __shared__ float2 sines[];   // [at_a_time][pairs], then [teams][head_dim] floats
  typedef NormUnit<T, E, HALF> Unit;
  const NormArgs& a = k.n;
  float* sums = reinterpret_cast<float*>(sines + a.at_a_time * a.pairs);
  const int lane = threadIdx.x & (a.lanes - 1), team = threadIdx.x >> a.log_lanes, teams = kNormThreads >> a.log_lanes;
  int tensor = 0;
  while ((int)blockIdx.x >= k.first[tensor + 1]) ++tensor;
  const int at = blockIdx.x - k.first[tensor], group = k.by_splits[tensor].of(at), split = at - group * k.splits[tensor], heads = k.group_heads[tensor];
  const int64_t begin = split * k.tokens_each[tensor], end = begin + k.tokens_each[tensor] < a.all ? begin + k.tokens_each[tensor] : a.all;
  const Heads &from = a.x[tensor], &grad = a.g[tensor], &to = a.out[tensor];
  const float by = 1.0f / (float)a.head_dim;
  const bool wanted = k.grad_weights[tensor] != nullptr;
  Unit w, add;
#pragma unroll
  for (int e = 0; e < Unit::N; ++e) add.v[e] = 0.f;
  if (ONE && lane < a.units) w.read_weight(a, tensor, group, lane);
  if (!ONE && wanted)
    for (int i = threadIdx.x; i < teams * a.head_dim; i += kNormThreads) sums[i] = 0.f;      // (barrier below)
  struct Row {
    const T *from, *grad;
    T* to;
    int tok;
    Unit x, g;
  };
  for (int64_t first = begin; first < end; first += a.at_a_time) {
    const int n = (int)(end - first < a.at_a_time ? end - first : a.at_a_time), rows = n * heads;
    auto find = [&](int i, Row& r) {
      r.tok = k.by_group[tensor].of(i);
      const int head = group * (heads == 1 ? 1 : 0) + (i - r.tok * heads);
      const uint32_t at = (uint32_t)(first + r.tok), b = a.by_tokens.of(at), t = at - b * a.tokens;
      r.from = reinterpret_cast<const T*>(from.data) + b * from.batch_stride + t * from.token_stride + head * from.head_stride;
      r.grad = reinterpret_cast<const T*>(grad.data) + b * grad.batch_stride + t * grad.token_stride + head * grad.head_stride;
      r.to = reinterpret_cast<T*>(to.data) + b * to.batch_stride + t * to.token_stride + head * to.head_stride;
      if (ONE && lane < a.units) {
        r.x.read(a, r.from, lane);
        r.g.read(a, r.grad, lane);
      }
    };
    Row row;
    if (team < rows) find(team, row);
    fill_sines(a, first, n, sines);
    __syncthreads();
    for (int i = team; i < rows; i += teams) {
      Row next;
      if (i + teams < rows) find(i + teams, next);
      const float2* cs = sines + row.tok * a.pairs;
      float sum = 0.f, dot = 0.f;
      for (int u = lane; u < a.units; u += a.lanes) {
        if (!ONE) {
          row.x.read(a, row.from, u);
          row.g.read(a, row.grad, u);
          w.read_weight(a, tensor, group, u);
        }
        row.g.template turn<true>(a, cs, u);
#pragma unroll
        for (int e = 0; e < Unit::N; ++e) {
          sum = __builtin_fmaf(row.x.v[e], row.x.v[e], sum);
          dot = __builtin_fmaf(row.g.v[e] * w.v[e], row.x.v[e], dot);
        }
      }
      sum = team_all(sum, a.lanes, plus);
      dot = team_all(dot, a.lanes, plus);
      const float r = 1.0f / __builtin_sqrtf(sum * by + a.eps), less = r * r * (dot * by);
      for (int u = lane; u < a.units; u += a.lanes) {
        if (!ONE) {
          row.x.read(a, row.from, u);
          row.g.read(a, row.grad, u);
          row.g.template turn<true>(a, cs, u);
          w.read_weight(a, tensor, group, u);
          if (wanted) {
            float* mine = sums + team * a.head_dim + Unit::place(a, u);
#pragma unroll
            for (int e = 0; e < Unit::N; ++e)
              if (e < E || u < a.turned) mine[e < E ? e : (HALF ? a.pairs : 1) + e - E] += row.g.v[e] * (row.x.v[e] * r);
          }
        }
        Unit out;
#pragma unroll
        for (int e = 0; e < Unit::N; ++e) {
          if (ONE) add.v[e] = __builtin_fmaf(row.g.v[e], row.x.v[e] * r, add.v[e]);
          out.v[e] = r * (row.g.v[e] * w.v[e] - row.x.v[e] * less);
        }
        out.write(a, row.to, u);
      }
      row = next;
    }
    __syncthreads();   // the next tokens' sines take the place of these
  }
  if (!wanted) return;
  if (ONE && lane < a.units) {
    float* mine = sums + team * a.head_dim + Unit::place(a, lane);
#pragma unroll
    for (int e = 0; e < Unit::N; ++e)
      if (e < E || lane < a.turned) mine[e < E ? e : (HALF ? a.pairs : 1) + e - E] = add.v[e];
  }
  __syncthreads();
  for (int d = threadIdx.x; d < a.head_dim; d += kNormThreads) {
    float s = 0.f;
    for (int t = 0; t < teams; ++t) s += sums[t * a.head_dim + d];
    k.parts[(int64_t)blockIdx.x * a.head_dim + d] = s;
  }
}

// The parts of a weight's gradient meet: a workgroup to 64 elements of a weight, its wavefronts take parts in turns.
constexpr int kNormJoin = 1024;
template <typename W>
__global__ void __launch_bounds__(kNormJoin) norm_rope_join_kernel(const NormBackArgs k, int pieces) {
  __shared__ float sums[kNormJoin / 64][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int weight = blockIdx.x / pieces, tensor = 0;
  const int d = (blockIdx.x - weight * pieces) * 64 + lane;
  while (weight >= k.groups_end[tensor]) ++tensor;
  if (tensor > 0) weight -= k.groups_end[tensor - 1];
  if (k.grad_weights[tensor] == nullptr) return;
  const int splits = k.splits[tensor];
  float s = 0.f;
  if (d < k.n.head_dim) {
    const float* from = k.parts + (int64_t)(k.first[tensor] + weight * splits) * k.n.head_dim + d;
#pragma unroll 4
    for (int i = wave; i < splits; i += kNormJoin / 64) s += from[(int64_t)i * k.n.head_dim];
  }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave > 0 || d >= k.n.head_dim) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < kNormJoin / 64; ++i) s += sums[i][lane];
  static_cast<W*>(k.grad_weights[tensor])[weight * k.n.weight_strides[tensor] + d] = (W)s;
}

}  // namespace dpllm
