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
  Divide by_tokens;
  int64_t all;                  // batch * tokens
  int tokens, heads, head_dim, pairs, rotary, units, turned, lanes, log_lanes, heads_each, weight_dtype;
  float eps, scale;
};

// What a lane has of a head: E elements, or where the two of a pair lie apart (HALF: half the rotated part; E = 1: neighbours) E and those E that go with them.
// Units from `turned` on are not rotated; where pairs lie apart they have their E elements twice, which saves the branches and does no harm but in sums.
template <typename T, int E, bool HALF>
struct NormUnit {
  static constexpr bool APART = HALF || E == 1;
  static constexpr int N = APART ? 2 * E : E;
  float v[N];
  struct Spot {      // where a unit lies
    int at, apart;
    bool turned;
  };
  __device__ __forceinline__ static Spot spot(const NormArgs& a, int u) {
    const bool turned = u < a.turned;
    return {turned ? u * (APART && !HALF ? 2 : E) : a.rotary + (u - a.turned) * E, turned ? (HALF ? a.pairs : 1) : 0, turned};
  }
  template <typename S>
  struct Raw {      // on its way from memory
    typedef S some __attribute__((ext_vector_type(E)));
    some a, b;
  };
  template <typename S>
  __device__ __forceinline__ static void ask(const S* head, const Spot& at, Raw<S>& x) {
    const S* p = head + at.at;
    x.a = *reinterpret_cast<const typename Raw<S>::some*>(p);
    if constexpr (APART) x.b = *reinterpret_cast<const typename Raw<S>::some*>(p + at.apart);
  }
  template <typename S>
  __device__ __forceinline__ void take(const Raw<S>& x) {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (float)x.a[e];
    if constexpr (APART)
#pragma unroll
      for (int e = 0; e < E; ++e) v[E + e] = (float)x.b[e];
  }
  template <typename S>
  __device__ __forceinline__ void read(const S* head, const Spot& at) {
    Raw<S> x;
    ask(head, at, x);
    take(x);
  }
  __device__ __forceinline__ void read_weight(const NormArgs& a, int tensor, int head, const Spot& at) {
    const void* w = a.weights[tensor];
    const int64_t from = head * a.weight_strides[tensor];
    if (w == nullptr) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = 1.f;
    } else if (a.weight_dtype == DPLLM_F32) {
      read(static_cast<const float*>(w) + from, at);
    } else if (a.weight_dtype == DPLLM_F16) {
      read(static_cast<const half_t*>(w) + from, at);
    } else {
      read(static_cast<const bfloat_t*>(w) + from, at);
    }
  }
  __device__ __forceinline__ void write(T* head, const Spot& at) const {
    typedef typename Raw<T>::some vec;
    T* p = head + at.at;
    vec x;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = (T)v[e];
    if constexpr (APART) {
      vec y;
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = (T)v[E + e];
      *reinterpret_cast<vec*>(p + at.apart) = y;
    }
    *reinterpret_cast<vec*>(p) = x;
  }
  // f(v) added up over a unit's elements, those that it has twice once.
  template <typename F>
  __device__ __forceinline__ static float sum(const Spot& at, F f) {
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s = f(e, s);
    if constexpr (APART) {
#pragma unroll
      for (int e = E; e < N; ++e) t = f(e, t);
      s += at.turned ? t : 0.f;
    }
    return s;
  }
  // The cosines and sines (times the scale) of a unit's pairs.
  static constexpr int P = HALF ? E : E > 1 ? E / 2 : 1;
  struct Angles {
    float2 of[P];
  };
  __device__ __forceinline__ static void read_angles(const float2* sines, int u, const Spot& at, Angles& x) {
    if (!at.turned) return;
#pragma unroll
    for (int e = 0; e < P; ++e) x.of[e] = sines[u * P + e];
  }
  // Turned by them; BACK: the transpose.
  template <bool BACK>
  __device__ __forceinline__ void turn(const Angles& x, const Spot& at) {
    if (!at.turned) return;
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const float2 f = x.of[e];
      const int i = APART ? e : 2 * e, j = APART ? E + e : 2 * e + 1;
      const float p = v[i], q = v[j], s = BACK ? -f.y : f.y;
      v[i] = p * f.x - q * s;
      v[j] = p * s + q * f.x;
    }
  }
};

// Sums over groups of L = 1, 2, ... 64 neighbouring lanes, the same L for all: steps that a group is too small for add nothing, which costs less than to branch round them.
struct Team {
  uint32_t masks[4];
  int lanes;
  __device__ __forceinline__ explicit Team(int lanes) : lanes(lanes) {
#pragma unroll
    for (int i = 0; i < 4; ++i) masks[i] = lanes > 1 << i ? ~0u : 0u;
  }
  template <int N>
  __device__ __forceinline__ void sums(float (&v)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __uint_as_float(other<0>(__float_as_uint(v[i])) & masks[0]);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __uint_as_float(other<1>(__float_as_uint(v[i])) & masks[1]);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __uint_as_float(other<2>(__float_as_uint(v[i])) & masks[2]);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __uint_as_float(other<3>(__float_as_uint(v[i])) & masks[3]);
    if (lanes > 16)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] += other<4>(v[i]);
        if (lanes > 32) v[i] += other<5>(v[i]);
      }
  }
};

// 1 / sqrt(v) to a step of its last bit; the instruction takes subnormal numbers for 0.
__device__ __forceinline__ float inverse_root(float v) {
  const bool small = v < 0x1p-96f;
  return __builtin_amdgcn_rsqf(small ? v * 0x1p64f : v) * (small ? 0x1p32f : 1.f);
}

// The sines of a token, made by a wavefront in LDS of its own, which no other reads.
__device__ __forceinline__ void fill_sines(const NormArgs& a, int position, float2* sines) {
  for (int i = threadIdx.x & 63; i < a.pairs; i += 64) {
    const double angle = (double)position * a.freqs[i];
    double t = angle * 0.15915494309189533577;   // 1 / (2 pi); as in rope_kernel.hpp
    t -= __builtin_rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    sines[i] = make_float2(c * a.scale, s * a.scale);
  }
}
__device__ __forceinline__ void met() {      // LDS that a wavefront's lanes have written is read by its others
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A wavefront takes a token and heads_each of its heads, a group of `lanes` lanes a head; so token, position and tensor are the same for a wavefront and what depends on them is done once, by scalar
// instructions.  ONE: a head has no more units than lanes, is read once, and kNormAtOnce heads of a group are on their way; else it is read again behind its sum.
// Bound by memory: 156 MB of three prompts of 2111 tokens, 40 + 8 heads of 128, in 29 us, 5.4 TB/s (a copy has 5.1; a call in a loop over other inputs each time 36.6).  With workgroups that took a few tokens' heads in turn,
// addresses and sines made lane by lane, it took 48 where this took 34.  One token takes 4 us of latency (position, sines, one head).
constexpr int kNormAtOnce = 2;
template <typename T, int E, bool HALF, bool ONE>
__global__ void __launch_bounds__(kNormThreads) norm_rope_kernel(const NormArgs a) {
  extern __shared__ float2 shared[];   // [wavefronts][pairs]
  typedef NormUnit<T, E, HALF> Unit;
  constexpr int AT = ONE ? kNormAtOnce : 1;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & (a.lanes - 1), team = (threadIdx.x & 63) >> a.log_lanes, teams = 64 >> a.log_lanes;
  const int first = blockIdx.y * a.heads_each, last = first + a.heads_each < a.heads ? first + a.heads_each : a.heads;
  const float by = 1.0f / (float)a.head_dim;
  const Team sums(a.lanes);
  float2* sines = shared + wave * a.pairs;
  const bool here = !ONE || lane < a.units;
  const int unit = lane < a.units ? lane : a.units - 1;      // (lanes without one read the last along)
  typename Unit::Spot spot = Unit::spot(a, unit);
  for (int64_t at = (int64_t)blockIdx.x * (kNormThreads / 64) + wave; at < a.all; at += (int64_t)gridDim.x * (kNormThreads / 64)) {
    const uint32_t b = a.by_tokens.of((uint32_t)at), t = (uint32_t)at - b * a.tokens;
    const int position = a.pairs > 0 ? a.positions[b * a.positions_stride + t] : 0;
    typename Unit::Angles angles;
    bool made = false;
    for (int tensor = 0, begin = 0; begin < last; begin = a.end[tensor++]) {
      const int low = first > begin ? first - begin : 0, high = (last < a.end[tensor] ? last : a.end[tensor]) - begin;
      if (low >= high) continue;
      const Heads &x_ = a.x[tensor], &out = a.out[tensor];
      const T* from = reinterpret_cast<const T*>(x_.data) + b * x_.batch_stride + t * x_.token_stride;
      T* to = reinterpret_cast<T*>(out.data) + b * out.batch_stride + t * out.token_stride;
      const int64_t from_stride = x_.head_stride, to_stride = out.head_stride;
      const bool each = a.weight_strides[tensor] != 0;
      typename Unit::template Raw<T> raw[AT];
      auto ask = [&](int head, typename Unit::template Raw<T>& r) { Unit::ask(from + (head < high ? head : high - 1) * from_stride, spot, r); };
      if (ONE)
#pragma unroll
        for (int k = 0; k < AT; ++k) ask(low + k * teams + team, raw[k]);
      Unit w;
      if (ONE && !each) w.read_weight(a, tensor, 0, spot);
      if (!made) {
        made = true;
        fill_sines(a, position, sines);
        met();
        if (ONE) Unit::read_angles(sines, unit, spot, angles);
      }
      for (int base = low; base < high; base += AT * teams) {
#pragma unroll
        for (int k = 0; k < AT; ++k) {
          const int head = base + k * teams + team;
          if (k > 0 && base + k * teams >= high) break;
          const T* mine = from + (head < high ? head : high - 1) * from_stride;
          Unit x;
          float sum[1] = {0.f};
          auto square = [&](int e, float s) { return __builtin_fmaf(x.v[e], x.v[e], s); };
          if (ONE) {
            x.take(raw[k]);
            ask(head + AT * teams, raw[k]);
            const float s = Unit::sum(spot, square);
            sum[0] = here ? s : 0.f;
          } else {
            for (int u = lane; u < a.units; u += a.lanes) {
              spot = Unit::spot(a, u);
              x.read(mine, spot);
              sum[0] += Unit::sum(spot, square);
            }
          }
          sums.sums(sum);
          const float norm = inverse_root(sum[0] * by + a.eps);
          auto finish = [&](int u) {
            if (!ONE) {
              spot = Unit::spot(a, u);
              x.read(mine, spot);
              Unit::read_angles(sines, u, spot, angles);
            }
            if (!ONE || each) w.read_weight(a, tensor, head < high ? head : high - 1, spot);
#pragma unroll
            for (int e = 0; e < Unit::N; ++e) x.v[e] = x.v[e] * norm * w.v[e];
            x.template turn<false>(angles, spot);
            if (here && head < high) x.write(to + head * to_stride, spot);
          };
          if (ONE)
            finish(unit);
          else
            for (int u = lane; u < a.units; u += a.lanes) finish(u);
        }
      }
    }
    met();   // the next token's sines take the place of these
  }
}

struct NormBackArgs {
  NormArgs n;
  float* parts;                      // [workgroup][weights of the workgroup][head_dim]
  int first[kNormTensors + 1];       // the first workgroup of a tensor
  int splits[kNormTensors];          // workgroups to a set of heads
  int set_heads[kNormTensors];       // heads of a set: all that share a weight, or one to a group of lanes
  int own[kNormTensors];             // weights of a set: 1, or one to a group of lanes
  int64_t parts_at[kNormTensors];    // where the tensor's parts are, in head_dims
  Divide by_splits[kNormTensors], by_own[kNormTensors];
  int64_t tokens_each[kNormTensors];      // tokens to a workgroup
  void* grad_weights[kNormTensors];
  int weights_end[kNormTensors];     // weights of the tensors up to and with this one
};

// A workgroup takes a stretch of tokens of a set of heads, its wavefronts every fourth token: a lane has the same elements of the same weight throughout and adds its gradient up in registers (in LDS
// where a lane has several units).  252 MB of 4 sequences of 2049 tokens, 32 + 8 heads of 128, in 52 us and 5 to join, 4.4 TB/s in all (a call in a loop 64); memory and instructions (300 to a head's step) both near
// their bounds: 73 us before roots, sums and loads were freed of branches.  Wavefronts and groups of lanes meet in LDS at the end, in their order, so the sum does not change from run to run.
template <typename T, int E, bool HALF, bool ONE>
__global__ void __launch_bounds__(kNormThreads) norm_rope_backward_kernel(const NormBackArgs k) {
  extern __shared__ float2 shared[];   // [wavefronts][pairs], then [wavefronts][groups of lanes][head_dim] floats
  typedef NormUnit<T, E, HALF> Unit;
  const NormArgs& a = k.n;
  constexpr int WAVES = kNormThreads / 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & (a.lanes - 1), team = (threadIdx.x & 63) >> a.log_lanes, teams = 64 >> a.log_lanes;
  float2* sines = shared + wave * a.pairs;
  float* added = reinterpret_cast<float*>(shared + WAVES * a.pairs);
  float* mine = added + (wave * teams + team) * a.head_dim;
  int tensor = 0;
  while ((int)blockIdx.x >= k.first[tensor + 1]) ++tensor;
  const int at = blockIdx.x - k.first[tensor], set = k.by_splits[tensor].of(at), split = at - set * k.splits[tensor], own = k.own[tensor];
  const int all_heads = a.end[tensor] - (tensor > 0 ? a.end[tensor - 1] : 0), low = set * k.set_heads[tensor];
  const int high = low + k.set_heads[tensor] < all_heads ? low + k.set_heads[tensor] : all_heads;
  const int64_t begin = split * k.tokens_each[tensor] + wave, end = (split + 1) * k.tokens_each[tensor] < a.all ? (split + 1) * k.tokens_each[tensor] : a.all;
  const Heads &x_ = a.x[tensor], &g_ = a.g[tensor], &out_ = a.out[tensor];
  const float by = 1.0f / (float)a.head_dim;
  const bool wanted = k.grad_weights[tensor] != nullptr, here = !ONE || lane < a.units;
  const Team sums(a.lanes);
  const int weight = own > 1 && low + team < high ? low + team : low;      // (a shared one lies at 0 whatever its number)
  const int unit = lane < a.units ? lane : a.units - 1;                    // (lanes without one read the last along)
  typename Unit::Spot spot = Unit::spot(a, unit);
  Unit w, add;
#pragma unroll
  for (int e = 0; e < Unit::N; ++e) add.v[e] = 0.f;
  if (ONE) w.read_weight(a, tensor, weight, spot);
  if (!ONE && wanted)
    for (int i = lane; i < a.head_dim; i += a.lanes) mine[i] = 0.f;
  struct Place {      // of a token
    const T *from, *grad;
    T* to;
    int position;
  };
  auto find = [&](int64_t token) {
    const uint32_t b = a.by_tokens.of((uint32_t)token), t = (uint32_t)token - b * a.tokens;
    Place p;
    p.from = reinterpret_cast<const T*>(x_.data) + b * x_.batch_stride + t * x_.token_stride;
    p.grad = reinterpret_cast<const T*>(g_.data) + b * g_.batch_stride + t * g_.token_stride;
    p.to = reinterpret_cast<T*>(out_.data) + b * out_.batch_stride + t * out_.token_stride;
    p.position = a.pairs > 0 ? a.positions[b * a.positions_stride + t] : 0;
    return p;
  };
  typename Unit::template Raw<T> raw_x, raw_g;
  auto ask = [&](const Place& p, int head) {
    if (!ONE) return;
    const int h = head < high ? head : high - 1;
    Unit::ask(p.from + h * x_.head_stride, spot, raw_x);
    Unit::ask(p.grad + h * g_.head_stride, spot, raw_g);
  };
  Place next{};
  if (begin < end) {
    next = find(begin);
    ask(next, low + team);
  }
  for (int64_t token = begin; token < end; token += WAVES) {
    const Place place = next;
    if (token + WAVES < end) next = find(token + WAVES);
    typename Unit::Angles angles;
    fill_sines(a, place.position, sines);
    met();
    if (ONE) Unit::read_angles(sines, unit, spot, angles);
    for (int base = low; base < high; base += teams) {
      const int head = base + team, h = head < high ? head : high - 1;
      const bool last = base + teams >= high;
      Unit x, g;
      if (ONE) {
        x.take(raw_x);
        g.take(raw_g);
        if (!last || token + WAVES < end) ask(last ? next : place, last ? low + team : head + teams);
      }
      float both[2] = {0.f, 0.f};
      auto measure = [&] {
        g.template turn<true>(angles, spot);
        both[0] += Unit::sum(spot, [&](int e, float s) { return __builtin_fmaf(x.v[e], x.v[e], s); });
        both[1] += Unit::sum(spot, [&](int e, float s) { return __builtin_fmaf(g.v[e] * w.v[e], x.v[e], s); });
      };
      auto fetch = [&](int u) {
        spot = Unit::spot(a, u);
        x.read(place.from + h * x_.head_stride, spot);
        g.read(place.grad + h * g_.head_stride, spot);
        w.read_weight(a, tensor, weight, spot);
        Unit::read_angles(sines, u, spot, angles);
      };
      if (ONE) {
        measure();
        both[0] = here ? both[0] : 0.f;
        both[1] = here ? both[1] : 0.f;
      } else {
        for (int u = lane; u < a.units; u += a.lanes) {
          fetch(u);
          measure();
        }
      }
      sums.sums(both);
      const float r = inverse_root(both[0] * by + a.eps), less = r * r * (both[1] * by);
      if (head >= high) continue;
      auto finish = [&] {
        Unit out;
#pragma unroll
        for (int e = 0; e < Unit::N; ++e) {
          const float y = g.v[e] * r;
          if (ONE) add.v[e] = __builtin_fmaf(y, x.v[e], add.v[e]);
          out.v[e] = __builtin_fmaf(-less * r, x.v[e], y * w.v[e]);
        }
        if (here) out.write(place.to + h * out_.head_stride, spot);
      };
      if (ONE) {
        finish();
      } else {
        for (int u = lane; u < a.units; u += a.lanes) {
          fetch(u);
          g.template turn<true>(angles, spot);
          if (wanted) {
            float* to = mine + spot.at;
#pragma unroll
            for (int e = 0; e < Unit::N; ++e)
              if (e < E || spot.turned) to[e < E ? e : (HALF ? a.pairs : 1) + e - E] += g.v[e] * (x.v[e] * r);
          }
          finish();
        }
      }
    }
    met();   // the next token's sines take the place of these
  }
  if (!wanted) return;
  if (ONE && here) {
    float* to = mine + spot.at;
#pragma unroll
    for (int e = 0; e < Unit::N; ++e)
      if (e < E || spot.turned) to[e < E ? e : (HALF ? a.pairs : 1) + e - E] = add.v[e];
  }
  __syncthreads();
  float* parts = k.parts + (k.parts_at[tensor] + (int64_t)at * own) * a.head_dim;
  for (int i = threadIdx.x; i < own * a.head_dim; i += kNormThreads) {
    float s = 0.f;
    if (own == 1)
      for (int t = 0; t < WAVES * teams; ++t) s += added[t * a.head_dim + i];
    else
      for (int t = 0; t < WAVES; ++t) s += added[t * teams * a.head_dim + i];      // (own = teams: weight after weight, as the sums lie)
    parts[i] = s;
  }
}

// The parts of a weight's gradient meet: a workgroup to 16 elements of a weight, 64 parts at a time.
constexpr int kNormJoin = 1024, kNormColumns = 16;
template <typename W>
__global__ void __launch_bounds__(kNormJoin) norm_rope_join_kernel(const NormBackArgs k, int pieces) {
  __shared__ float sums[kNormJoin / 64][kNormColumns];
  int weight = blockIdx.x / pieces, tensor = 0;
  const int column = threadIdx.x % kNormColumns, d = (blockIdx.x - weight * pieces) * kNormColumns + column;
  while (weight >= k.weights_end[tensor]) ++tensor;
  if (tensor > 0) weight -= k.weights_end[tensor - 1];
  if (k.grad_weights[tensor] == nullptr) return;
  const int splits = k.splits[tensor], own = k.own[tensor], set = k.by_own[tensor].of(weight);
  float s = 0.f;
  if (d < k.n.head_dim) {
    const float* from = k.parts + (k.parts_at[tensor] + (int64_t)set * splits * own + (weight - set * own)) * k.n.head_dim + d;
#pragma unroll 4
    for (int i = threadIdx.x / kNormColumns; i < splits; i += kNormJoin / kNormColumns) s += from[(int64_t)i * own * k.n.head_dim];
  }
  s += __shfl_xor(s, 16);
  s += __shfl_xor(s, 32);
  if ((threadIdx.x & 63) < kNormColumns) sums[threadIdx.x >> 6][column] = s;
  __syncthreads();
  if (threadIdx.x >= kNormColumns || d >= k.n.head_dim) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < kNormJoin / 64; ++i) s += sums[i][column];
  static_cast<W*>(k.grad_weights[tensor])[weight * k.n.weight_strides[tensor] + d] = (W)s;
}

}  // namespace dpllm
