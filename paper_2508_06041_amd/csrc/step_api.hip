// Host side of dpllm_norm_rope, its gradient and dpllm_sample: argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "norm_rope_kernel.hpp"
#include "sample_kernels.hpp"
#include "token_host.hpp"

using namespace dpllm;

namespace {

// What both directions of the norms check and fill alike.  others: one or two more views of each tensor.
struct NormSetup {
  NormArgs a;
  bool half;
  int elements;      // of a unit: pieces of 16 bytes, of 8 or single
};

int setup_norm(const char* who, NormSetup* made, const dpllm_heads* x, const dpllm_heads* g, const dpllm_heads* out, const int* heads, const void* const* weights,
               const int64_t* weight_strides, int weight_dtype, float eps, int tensors, int batch, int tokens, int head_dim, int dtype, int rotary_dim, int layout,
               const double* freqs, float scale, const int32_t* positions, int64_t positions_stride) {
  if (!x || !g || !out || !heads) return refuse(DPLLM_EINVAL, "%s: a pointer is NULL", who);
  if (tensors < 1 || tensors > DPLLM_MAX_TENSORS) return refuse(DPLLM_ESHAPE, "%s: %d tensors, takes 1 to %d", who, tensors, DPLLM_MAX_TENSORS);
  if (dtype < DPLLM_F16 || dtype > DPLLM_F32) return refuse(DPLLM_EINVAL, "%s: unknown dtype %d", who, dtype);
  if (weights && (weight_dtype < DPLLM_F16 || weight_dtype > DPLLM_F32)) return refuse(DPLLM_EINVAL, "%s: unknown weight_dtype %d", who, weight_dtype);
  if (weights && !weight_strides) return refuse(DPLLM_EINVAL, "%s: weight_strides is NULL", who);
  if (layout != DPLLM_ROPE_HALF && layout != DPLLM_ROPE_INTERLEAVED) return refuse(DPLLM_EINVAL, "%s: unknown layout %d", who, layout);
  if (!(eps >= 0.f) || std::isinf(eps)) return refuse(DPLLM_EINVAL, "%s: eps has to be finite and not negative", who);
  if (batch < 0 || tokens < 0 || (int64_t)batch * tokens > INT32_MAX) return refuse(DPLLM_ESHAPE, "%s: %d sequences of %d tokens", who, batch, tokens);
  if (head_dim < 1 || head_dim > DPLLM_MAX_HEAD_DIM || rotary_dim < 0 || rotary_dim % 2 || rotary_dim > head_dim)
    return refuse(DPLLM_ESHAPE, "%s: rotary_dim %d of head_dim %d (even, head_dim at most %d)", who, rotary_dim, head_dim, DPLLM_MAX_HEAD_DIM);
  const bool some = batch > 0 && tokens > 0;
  if (rotary_dim > 0 && some && (!freqs || !positions)) return refuse(DPLLM_EINVAL, "%s: freqs or positions is NULL", who);
  const int es = dtype == DPLLM_F32 ? 4 : 2, ws = weight_dtype == DPLLM_F32 ? 4 : 2, wide = 16 / es;
  made->half = layout == DPLLM_ROPE_HALF && rotary_dim > 0;
  auto whole = [&](int e) { return rotary_dim % (made->half ? 2 * e : e) == 0 && (head_dim - rotary_dim) % e == 0; };
  bool vector = true;
  NormArgs& a = made->a;
  a = {};
  int64_t all_heads = 0;
  for (int i = 0; i < tensors; ++i) {
    if (heads[i] < 1) return refuse(DPLLM_ESHAPE, "%s: tensor %d has %d heads", who, i, heads[i]);
    if (some && (!x[i].data || !g[i].data || !out[i].data)) return refuse(DPLLM_EINVAL, "%s: tensor %d is NULL", who, i);
    if (((uintptr_t)x[i].data | (uintptr_t)g[i].data | (uintptr_t)out[i].data) % es) return refuse(DPLLM_EINVAL, "%s: tensor %d is not aligned to its elements", who, i);
    all_heads += heads[i];
    if (all_heads * head_dim > (1 << 24)) return refuse(DPLLM_ESHAPE, "%s: %lld heads of %d", who, (long long)all_heads, head_dim);
    a.end[i] = (int)all_heads;
    const dpllm_heads views[3] = {reached(x[i], batch, tokens, heads[i]), reached(g[i], batch, tokens, heads[i]), reached(out[i], batch, tokens, heads[i])};
    a.x[i] = view(views[0]);
    a.g[i] = view(views[1]);
    a.out[i] = view(views[2]);
    for (const dpllm_heads& v : views) vector = vector && pieces(v, es);
    a.weights[i] = weights ? weights[i] : nullptr;
    a.weight_strides[i] = weights ? weight_strides[i] : 0;
    if ((uintptr_t)a.weights[i] % ws) return refuse(DPLLM_EINVAL, "%s: weight %d is not aligned to its elements", who, i);
    vector = vector && (uintptr_t)a.weights[i] % 16 == 0 && a.weight_strides[i] * ws % 16 == 0;
  }
  // Eight elements to a lane at most: with sixteen (two pieces of 16 bytes where pairs lie apart) the gradient has registers for three wavefronts to a SIMD and took 86.6 us, with eight 73.3.
  const int most = made->half ? 4 : wide, e = !vector ? 1 : whole(most) ? most : whole(wide / 2) ? wide / 2 : 1;
  made->elements = e;
  a.freqs = freqs;
  a.positions = positions;
  a.positions_stride = positions_stride;
  a.all = (int64_t)batch * tokens;
  a.tokens = tokens;
  a.heads = (int)all_heads;
  a.head_dim = head_dim;
  a.pairs = rotary_dim / 2;
  a.rotary = rotary_dim;
  a.turned = made->half ? a.pairs / e : a.pairs / (e > 1 ? e / 2 : 1);
  a.units = a.turned + (head_dim - rotary_dim) / e;
  while ((1 << a.log_lanes) < std::min(a.units, 64)) ++a.log_lanes;
  a.lanes = 1 << a.log_lanes;
  a.weight_dtype = weight_dtype;
  a.eps = eps;
  a.scale = scale;
  a.by_tokens = Divide::by(std::max(tokens, 1));
  return DPLLM_OK;
}

// f(type, elements, half, one) with the constants that belong to the arguments
template <typename F>
void choose_norm(const NormSetup& s, int dtype, F f) {
  auto by_one = [&](auto type, auto e, auto half) {
    s.a.units <= s.a.lanes ? f(type, e, half, std::true_type()) : f(type, e, half, std::false_type());
  };
  auto by_half = [&](auto type, auto e) { s.half ? by_one(type, e, std::true_type()) : by_one(type, e, std::false_type()); };
  auto by_e = [&](auto type) {
    constexpr int kWide = 16 / sizeof(type);
    if constexpr (kWide == 8)
      if (s.elements == kWide) by_one(type, std::integral_constant<int, kWide>(), std::false_type());
    if constexpr (kWide == 4)
      if (s.elements == kWide) by_half(type, std::integral_constant<int, kWide>());
    if (s.elements == kWide / 2) by_half(type, std::integral_constant<int, kWide / 2>());
    if (s.elements == 1) by_half(type, std::integral_constant<int, 1>());
  };
  if (dtype == DPLLM_F16) by_e(half_t());
  if (dtype == DPLLM_BF16) by_e(bfloat_t());
  if (dtype == DPLLM_F32) by_e(float());
}

// How the gradient's work is dealt out: workgroups to each set of heads, teams groups of lanes to a wavefront.
struct NormSplit {
  int splits[kNormTensors], first[kNormTensors + 1], set_heads[kNormTensors], own[kNormTensors], weights_end[kNormTensors];
  int64_t tokens_each[kNormTensors], parts_at[kNormTensors], parts;
};
constexpr int kNormGroups = 1280;      // five to a compute unit, as many as registers allow: 57 us (with the join) for the gradient of 4 sequences of 2049 tokens, 32 + 8 heads of 128; 1024: 58, 1536: 64, 2048: 61
NormSplit split_norm(const int* heads, const int64_t* weight_strides, int tensors, int64_t all, int teams) {
  NormSplit s{};
  int64_t all_heads = 0;
  for (int i = 0; i < tensors; ++i) all_heads += heads[i];
  for (int i = 0; i < tensors; ++i) {
    const bool each = weight_strides && weight_strides[i] != 0;
    s.own[i] = each ? teams : 1;
    s.set_heads[i] = each ? teams : heads[i];
    const int sets = (heads[i] + s.set_heads[i] - 1) / s.set_heads[i];
    // about kNormGroups workgroups in all, each of at least 16 heads
    const int64_t wish = std::max<int64_t>(1, (int64_t)kNormGroups * std::min(s.set_heads[i], heads[i]) / all_heads), most = std::max<int64_t>(1, all * s.set_heads[i] / 16);
    s.tokens_each[i] = std::max<int64_t>(1, (all + std::min(wish, most) - 1) / std::min(wish, most));
    s.splits[i] = (int)std::max<int64_t>(1, (all + s.tokens_each[i] - 1) / s.tokens_each[i]);
    s.first[i + 1] = s.first[i] + sets * s.splits[i];
    s.parts_at[i] = s.parts;
    s.parts += (int64_t)sets * s.splits[i] * s.own[i];
    s.weights_end[i] = (each ? heads[i] : 1) + (i > 0 ? s.weights_end[i - 1] : 0);
  }
  for (int i = tensors; i < kNormTensors; ++i) s.first[i + 1] = s.first[i];
  return s;
}

// The workspace of a draw: tops of the chunks, then their histograms.
struct SampleBytes {
  int chunks;
  size_t tops, bytes;
};
SampleBytes sample_bytes(int rows, int vocabulary, int dtype) {
  const int e = dtype == DPLLM_F32 ? 4 : 8, chunk = kVerThreads * kVerPieces * e;
  SampleBytes s;
  s.chunks = (int)(((int64_t)vocabulary + e - 1 + chunk - 1) / chunk);      // a row may start up to e - 1 elements behind a 16-byte boundary
  s.tops = ((size_t)rows * s.chunks * sizeof(SampleTop) + 15) / 16 * 16;
  s.bytes = s.tops + (size_t)rows * s.chunks * kSampleBins * sizeof(unsigned long long);
  return s;
}

int check_sample(const char* who, int rows, int vocabulary, int dtype) {
  if (dtype < DPLLM_F16 || dtype > DPLLM_F32) return refuse(DPLLM_EINVAL, "%s: unknown dtype %d", who, dtype);
  if (rows < 0 || rows > 65536) return refuse(DPLLM_ESHAPE, "%s: %d rows (at most 65536)", who, rows);
  // (a running sum over the chunks takes two to a thread)
  if (vocabulary < 1 || vocabulary > (1 << 22)) return refuse(DPLLM_ESHAPE, "%s: a vocabulary of %d words (1 to 2^22)", who, vocabulary);
  if ((int64_t)rows * sample_bytes(1, vocabulary, dtype).chunks > 0xffffff) return refuse(DPLLM_ESHAPE, "%s: %d rows of %d words are too many at once", who, rows, vocabulary);
  return DPLLM_OK;
}

template <typename T>
void launch_sample(const SampleArgs& a, hipStream_t s) {
  const dim3 groups(a.rows < 8 ? a.rows : (a.rows + 7) / 8 * 8, a.chunks);
  hipLaunchKernelGGL(sample_tops_kernel<T>, groups, dim3(kVerThreads), 0, s, a);
  hipLaunchKernelGGL(sample_bins_kernel<T>, groups, dim3(kVerThreads), 0, s, a);
  hipLaunchKernelGGL(sample_choose_kernel<T>, dim3(a.rows), dim3(kSampleThreads), 0, s, a);
}

}  // namespace

extern "C" {

int dpllm_norm_rope(const dpllm_heads* x, const dpllm_heads* out, const int* heads, const void* const* weights, const int64_t* weight_strides, int weight_dtype,
                    float eps, int tensors, int batch, int tokens, int head_dim, int dtype, int rotary_dim, int layout, const double* freqs_dev, float scale,
                    const int32_t* positions_dev, int64_t positions_stride, void* stream) {
  const char* who = "dpllm_norm_rope";
  NormSetup s;
  if (int rc = setup_norm(who, &s, x, x, out, heads, weights, weight_strides, weight_dtype, eps, tensors, batch, tokens, head_dim, dtype, rotary_dim, layout, freqs_dev, scale,
                          positions_dev, positions_stride))
    return rc;
  NormArgs& a = s.a;
  if (a.all == 0) return DPLLM_OK;
  // a token's heads in one wavefront if tokens alone give the chip wavefronts enough, else in several
  const int teams = 64 >> a.log_lanes, waves = kNormThreads / 64, rounds = (a.heads + teams - 1) / teams, chunks = (int)std::min<int64_t>(rounds, std::max<int64_t>(1, 4096 / a.all));
  a.heads_each = (rounds + chunks - 1) / chunks * teams;
  const dim3 grid((unsigned)std::min<int64_t>((a.all + waves - 1) / waves, 1 << 20), (unsigned)((a.heads + a.heads_each - 1) / a.heads_each));
  choose_norm(s, dtype, [&](auto type, auto e, auto half, auto one) {
    hipLaunchKernelGGL((norm_rope_kernel<decltype(type), decltype(e)::value, decltype(half)::value, decltype(one)::value>), grid, dim3(kNormThreads),
                       sizeof(float2) * waves * a.pairs, (hipStream_t)stream, a);
  });
  return launched(who);
}

int dpllm_norm_rope_backward_workspace_bytes(const int* heads, const int64_t* weight_strides, int tensors, int batch, int tokens, int head_dim, size_t* bytes) {
  const char* who = "dpllm_norm_rope_backward_workspace_bytes";
  if (!heads || !bytes) return refuse(DPLLM_EINVAL, "%s: a pointer is NULL", who);
  if (tensors < 1 || tensors > DPLLM_MAX_TENSORS) return refuse(DPLLM_ESHAPE, "%s: %d tensors, takes 1 to %d", who, tensors, DPLLM_MAX_TENSORS);
  if (batch < 0 || tokens < 0 || (int64_t)batch * tokens > INT32_MAX) return refuse(DPLLM_ESHAPE, "%s: %d sequences of %d tokens", who, batch, tokens);
  int64_t all_heads = 0;
  for (int i = 0; i < tensors; ++i) {
    if (heads[i] < 1) return refuse(DPLLM_ESHAPE, "%s: tensor %d has %d heads", who, i, heads[i]);
    all_heads += heads[i];
  }
  if (head_dim < 1 || head_dim > DPLLM_MAX_HEAD_DIM || all_heads * head_dim > (1 << 24)) return refuse(DPLLM_ESHAPE, "%s: %lld heads of %d", who, (long long)all_heads, head_dim);
  const int64_t all = (int64_t)batch * tokens;
  // the groups of lanes of a wavefront depend on types and strides as well, and are at most those of 16 elements to a lane
  int64_t parts = 0;
  for (int teams = 1; teams <= std::min(64, std::max(1, 1024 / head_dim)); teams *= 2) parts = std::max(parts, split_norm(heads, weight_strides, tensors, all, teams).parts);
  *bytes = all == 0 ? 0 : (size_t)parts * head_dim * sizeof(float);
  return DPLLM_OK;
}

int dpllm_norm_rope_backward(const dpllm_heads* x, const dpllm_heads* grads, const dpllm_heads* grad_x, const int* heads, const void* const* weights,
                             void* const* grad_weights, const int64_t* weight_strides, int weight_dtype, float eps, int tensors, int batch, int tokens, int head_dim, int dtype,
                             int rotary_dim, int layout, const double* freqs_dev, float scale, const int32_t* positions_dev, int64_t positions_stride, void* ws_dev,
                             size_t ws_bytes, void* stream) {
  const char* who = "dpllm_norm_rope_backward";
  NormSetup s;
  if (int rc = setup_norm(who, &s, x, grads, grad_x, heads, weights, weight_strides, weight_dtype, eps, tensors, batch, tokens, head_dim, dtype, rotary_dim, layout, freqs_dev,
                          scale, positions_dev, positions_stride))
    return rc;
  bool wanted = false;
  for (int i = 0; i < tensors; ++i) {
    if (!grad_weights || !grad_weights[i]) continue;
    wanted = true;
    if (!weights || !weights[i]) return refuse(DPLLM_EINVAL, "%s: the gradient of weight %d is wanted, which is NULL", who, i);
    if ((uintptr_t)grad_weights[i] % (weight_dtype == DPLLM_F32 ? 4 : 2)) return refuse(DPLLM_EINVAL, "%s: the gradient of weight %d is not aligned to its elements", who, i);
  }
  const NormArgs& a = s.a;
  if (a.all == 0 && !wanted) return DPLLM_OK;
  const NormSplit split = split_norm(heads, weights ? weight_strides : nullptr, tensors, a.all, 64 >> a.log_lanes);
  const size_t need = a.all == 0 || !wanted ? 0 : (size_t)split.parts * head_dim * sizeof(float);
  if (need > 0 && (!ws_dev || ws_bytes < need || (uintptr_t)ws_dev % 16)) return refuse(DPLLM_ESTATE, "%s: needs a workspace of %zu bytes, aligned to 16", who, need);
  NormBackArgs k{};
  k.n = a;
  k.parts = (float*)ws_dev;
  for (int i = 0; i < kNormTensors; ++i) {
    k.first[i + 1] = split.first[i + 1];
    k.splits[i] = a.all == 0 ? 0 : split.splits[i];
    k.set_heads[i] = std::max(split.set_heads[i], 1);
    k.own[i] = std::max(split.own[i], 1);
    k.parts_at[i] = split.parts_at[i];
    k.by_own[i] = Divide::by(k.own[i]);
    k.by_splits[i] = Divide::by(std::max(split.splits[i], 1));
    k.tokens_each[i] = split.tokens_each[i];
    k.grad_weights[i] = i < tensors && grad_weights ? grad_weights[i] : nullptr;
    k.weights_end[i] = i < tensors ? split.weights_end[i] : split.weights_end[tensors - 1];
  }
  if (a.all > 0) {
    const size_t lds = (kNormThreads / 64) * (sizeof(float2) * a.pairs + sizeof(float) * (64 >> a.log_lanes) * head_dim);
    choose_norm(s, dtype, [&](auto type, auto e, auto half, auto one) {
      hipLaunchKernelGGL((norm_rope_backward_kernel<decltype(type), decltype(e)::value, decltype(half)::value, decltype(one)::value>), dim3(split.first[tensors]),
                         dim3(kNormThreads), lds, (hipStream_t)stream, k);
    });
  }
  if (wanted) {
    const int each = (head_dim + kNormColumns - 1) / kNormColumns;
    const dim3 grid(split.weights_end[tensors - 1] * each), threads(kNormJoin);
    if (weight_dtype == DPLLM_F16) hipLaunchKernelGGL(norm_rope_join_kernel<half_t>, grid, threads, 0, (hipStream_t)stream, k, each);
    if (weight_dtype == DPLLM_BF16) hipLaunchKernelGGL(norm_rope_join_kernel<bfloat_t>, grid, threads, 0, (hipStream_t)stream, k, each);
    if (weight_dtype == DPLLM_F32) hipLaunchKernelGGL(norm_rope_join_kernel<float>, grid, threads, 0, (hipStream_t)stream, k, each);
  }
  return launched(who);
}

int dpllm_sample_workspace_bytes(int rows, int vocabulary, int dtype, size_t* bytes) {
  const char* who = "dpllm_sample_workspace_bytes";
  if (!bytes) return refuse(DPLLM_EINVAL, "%s: bytes is NULL", who);
  if (int rc = check_sample(who, rows, vocabulary, dtype)) return rc;
  *bytes = sample_bytes(rows, vocabulary, dtype).bytes;
  return DPLLM_OK;
}

int dpllm_sample(int rows, int vocabulary, int dtype, const void* logits_dev, int64_t stride, const float* uniforms_dev, const float* temperature_dev,
                 const int32_t* top_k_dev, const float* top_p_dev, const float* min_p_dev, int32_t* words_dev, int32_t* kept_dev, void* ws_dev, size_t ws_bytes,
                 void* stream) {
  const char* who = "dpllm_sample";
  if (int rc = check_sample(who, rows, vocabulary, dtype)) return rc;
  if (rows == 0) return DPLLM_OK;
  if (!logits_dev || !uniforms_dev || !temperature_dev || !words_dev)
    return refuse(DPLLM_EINVAL, "%s: a pointer is NULL (top_k_dev, top_p_dev, min_p_dev and kept_dev may be)", who);
  if ((uintptr_t)logits_dev % (dtype == DPLLM_F32 ? 4 : 2)) return refuse(DPLLM_EINVAL, "%s: the rows are not aligned to their elements", who);
  const SampleBytes space = sample_bytes(rows, vocabulary, dtype);
  if (!ws_dev || ws_bytes < space.bytes || (uintptr_t)ws_dev % 16) return refuse(DPLLM_ESTATE, "%s: needs a workspace of %zu bytes, aligned to 16", who, space.bytes);
  SampleArgs a{};
  a.logits = (const char*)logits_dev;
  a.stride = rows > 1 ? stride : 0;
  a.uniforms = uniforms_dev;
  a.temperature = temperature_dev;
  a.top_k = top_k_dev;
  a.top_p = top_p_dev;
  a.min_p = min_p_dev;
  a.words = words_dev;
  a.kept = kept_dev;
  a.tops = (SampleTop*)ws_dev;
  a.bins = (unsigned long long*)((char*)ws_dev + space.tops);
  a.rows = rows;
  a.vocabulary = vocabulary;
  a.chunks = space.chunks;
  if (dtype == DPLLM_F16) launch_sample<half_t>(a, (hipStream_t)stream);
  if (dtype == DPLLM_BF16) launch_sample<bfloat_t>(a, (hipStream_t)stream);
  if (dtype == DPLLM_F32) launch_sample<float>(a, (hipStream_t)stream);
  return launched(who);
}

}  // extern "C"
