// Host side of the calls around the linears that include/dpllm.h declares: argument checks and launches.  No kernel arithmetic lives here.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "append_kernel.hpp"
#include "rope_kernel.hpp"
#include "token_host.hpp"
#include "verify_kernels.hpp"

using namespace dpllm;

namespace {

template <typename T, int E>
void launch_rope(const RopeArgs& a, bool half, int blocks, size_t lds, hipStream_t stream) {
  if (half)
    hipLaunchKernelGGL((rope_kernel<T, E, true>), dim3(blocks), dim3(kRopeThreads), lds, stream, a);
  else
    hipLaunchKernelGGL((rope_kernel<T, E, false>), dim3(blocks), dim3(kRopeThreads), lds, stream, a);
}

// The workspace of a verification: the parts of the rows, the sums of what is left, what is known of the rows.
struct VerifySpace {
  int chunks;
  size_t parts, rest, bytes;
};

VerifySpace verify_space(int batch, int nodes, int vocabulary, int dtype, bool draft, int siblings) {
  const int e = dtype == DPLLM_F32 ? 4 : 8, chunk = kVerThreads * kVerPieces * e;
  VerifySpace s;
  s.chunks = (int)(((int64_t)vocabulary + e - 1 + chunk - 1) / chunk);      // a row may start up to e - 1 elements behind a 16-byte boundary
  const size_t all = (size_t)batch * nodes * s.chunks;
  s.parts = all * sizeof(VerifyPart) * (draft ? 2 : 1);
  s.rest = draft ? (all * siblings * sizeof(double) + 15) / 16 * 16 : 0;
  s.bytes = s.parts + s.rest + (draft ? (size_t)batch * nodes * sizeof(RowInfo) : 0);
  return s;
}

int check_verify(const char* who, int batch, int nodes, int vocabulary, int dtype, bool draft, int siblings) {
  if (dtype < DPLLM_F16 || dtype > DPLLM_F32) return refuse(DPLLM_EINVAL, "%s: unknown dtype %d", who, dtype);
  if (batch < 0 || batch > 65536 || nodes < 1 || nodes > DPLLM_MAX_NODES)
    return refuse(DPLLM_ESHAPE, "%s: %d sequences of %d nodes (at most 65536 of 1 to %d)", who, batch, nodes, DPLLM_MAX_NODES);
  if (vocabulary < 1 || vocabulary > (1 << 24)) return refuse(DPLLM_ESHAPE, "%s: a vocabulary of %d words (1 to 2^24)", who, vocabulary);
  if (draft && (siblings < 1 || siblings > DPLLM_MAX_NODES)) return refuse(DPLLM_ESHAPE, "%s: %d siblings (1 to %d)", who, siblings, DPLLM_MAX_NODES);
  if ((int64_t)batch * nodes * verify_space(1, 1, vocabulary, dtype, false, 1).chunks > 0xffffff)
    return refuse(DPLLM_ESHAPE, "%s: %d sequences of %d nodes with %d words are too many at once", who, batch, nodes, vocabulary);
  return DPLLM_OK;
}

template <typename T>
void launch_verify(const VerifyArgs& a, hipStream_t s) {
  const unsigned rows = (unsigned)a.batch * a.nodes;
  // three rounds of workgroups, whose next chunks come while they work: 640 rows (and 128 that are not read) of 128256 words in bf16 take 64 us with one workgroup to a row, 61 with two,
  // 54 with four, 56 with six, 61 with one to a chunk; few rows one to a chunk
  const int64_t all = (int64_t)rows * (a.draft ? 2 : 1);
  const int each = (int)std::min<int64_t>(a.chunks, (3000 + all - 1) / all);
  hipLaunchKernelGGL(verify_parts_kernel<T>, dim3(rows * each, a.draft ? 2 : 1), dim3(kVerThreads), 0, s, a, each, Divide::by(each));
  // few rows want a sum, so those that do are split finely: as many workgroups as fill the chip if one row in four does
  const int groups = std::max(1, std::min(a.chunks, (int)(16384 / rows)));
  for (int round = 0; a.draft && round < a.siblings; ++round) {
    hipLaunchKernelGGL(verify_rows_kernel<T>, dim3((rows + kVerThreads / 64 - 1) / (kVerThreads / 64)), dim3(kVerThreads), 0, s, a, round);
    hipLaunchKernelGGL(verify_rest_kernel<T>, dim3(rows * groups), dim3(kVerThreads), 0, s, a, round, groups);
  }
  hipLaunchKernelGGL(verify_choose_kernel<T>, dim3(a.batch), dim3(kVerChooseThreads), 0, s, a);
}

}  // namespace

extern "C" {

const char* dpllm_call_error(void) { return call_error(); }

int dpllm_rope_frequencies(int rotary_dim, double base, int scaling, double factor, double trained, double low, double high, double* freqs,
                           float* scale) {
  if (!freqs || !scale) return refuse(DPLLM_EINVAL, "dpllm_rope_frequencies: freqs or scale is NULL");
  if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > DPLLM_MAX_HEAD_DIM)
    return refuse(DPLLM_ESHAPE, "dpllm_rope_frequencies: rotary_dim %d is odd or outside [2, %d]", rotary_dim, DPLLM_MAX_HEAD_DIM);
  if (!(base > 1.0) || std::isinf(base)) return refuse(DPLLM_EINVAL, "dpllm_rope_frequencies: base has to be above 1 and finite");
  if (scaling < DPLLM_ROPE_PLAIN || scaling > DPLLM_ROPE_BANDS) return refuse(DPLLM_EINVAL, "dpllm_rope_frequencies: unknown scaling %d", scaling);
  if (scaling != DPLLM_ROPE_PLAIN && (!(factor >= 1.0) || std::isinf(factor)))
    return refuse(DPLLM_EINVAL, "dpllm_rope_frequencies: factor has to be at least 1 and finite");
  if (scaling == DPLLM_ROPE_NTK && rotary_dim == 2) return refuse(DPLLM_ESHAPE, "dpllm_rope_frequencies: NTK needs a rotary_dim above 2");
  if (scaling >= DPLLM_ROPE_YARN && (!(trained > 0.0) || std::isinf(trained) || !(low > 0.0) || !(high > low) || std::isinf(high)))
    return refuse(DPLLM_EINVAL, "dpllm_rope_frequencies: needs trained > 0 and high > low > 0");
  const double tau = 6.283185307179586476925;
  if (scaling == DPLLM_ROPE_NTK) base *= std::pow(factor, rotary_dim / (rotary_dim - 2.0));
  // the pairs that turn `high` and `low` times over the trained positions, by number; a ramp of no width is given a little
  const double lo = std::fmax(std::floor(rotary_dim * std::log(trained / (high * tau)) / (2 * std::log(base))), 0.0);
  double hi = std::fmin(std::ceil(rotary_dim * std::log(trained / (low * tau)) / (2 * std::log(base))), rotary_dim - 1.0);
  if (!(hi > lo)) hi = lo + 0.001;
  *scale = scaling == DPLLM_ROPE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / rotary_dim);
    double plain = 1.0;   // how much of the plain angle is left
    if (scaling == DPLLM_ROPE_LINEAR) plain = 0.0;
    if (scaling == DPLLM_ROPE_YARN) plain = 1.0 - std::fmin(std::fmax((i - lo) / (hi - lo), 0.0), 1.0);
    if (scaling == DPLLM_ROPE_BANDS) plain = std::fmin(std::fmax((trained * f / tau - low) / (high - low), 0.0), 1.0);
    freqs[i] = plain * f + (1.0 - plain) * f / (scaling == DPLLM_ROPE_PLAIN || scaling == DPLLM_ROPE_NTK ? 1.0 : factor);
  }
  return DPLLM_OK;
}

int dpllm_rope(const dpllm_heads* x, const dpllm_heads* out, const int* heads, int tensors, int batch, int tokens, int head_dim, int dtype,
               int rotary_dim, int layout, const double* freqs_dev, float scale, const int32_t* positions_dev, int64_t positions_stride, int inverse,
               void* stream) {
  if (!x || !out || !heads || !freqs_dev || (!positions_dev && batch > 0 && tokens > 0)) return refuse(DPLLM_EINVAL, "dpllm_rope: a pointer is NULL");
  if (tensors < 1 || tensors > DPLLM_MAX_TENSORS) return refuse(DPLLM_ESHAPE, "dpllm_rope: %d tensors, takes 1 to %d", tensors, DPLLM_MAX_TENSORS);
  if (dtype < DPLLM_F16 || dtype > DPLLM_F32) return refuse(DPLLM_EINVAL, "dpllm_rope: unknown dtype %d", dtype);
  if (layout != DPLLM_ROPE_HALF && layout != DPLLM_ROPE_INTERLEAVED) return refuse(DPLLM_EINVAL, "dpllm_rope: unknown layout %d", layout);
  if (batch < 0 || tokens < 0 || (int64_t)batch * tokens > INT32_MAX) return refuse(DPLLM_ESHAPE, "dpllm_rope: %d sequences of %d tokens", batch, tokens);
  if (head_dim < 2 || head_dim > DPLLM_MAX_HEAD_DIM || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > head_dim)
    return refuse(DPLLM_ESHAPE, "dpllm_rope: rotary_dim %d of head_dim %d (even, at least 2, head_dim at most %d)", rotary_dim, head_dim, DPLLM_MAX_HEAD_DIM);
  const int es = dtype == DPLLM_F32 ? 4 : 2, wide = 16 / es;
  const bool half = layout == DPLLM_ROPE_HALF;
  bool vector = rotary_dim % (half ? 2 * wide : wide) == 0 && (head_dim - rotary_dim) % wide == 0, same = true;
  RopeArgs a{};
  int64_t all_heads = 0;
  for (int i = 0; i < tensors; ++i) {
    if (heads[i] < 1) return refuse(DPLLM_ESHAPE, "dpllm_rope: tensor %d has %d heads", i, heads[i]);
    if (batch > 0 && tokens > 0 && (!x[i].data || !out[i].data)) return refuse(DPLLM_EINVAL, "dpllm_rope: tensor %d is NULL", i);
    if (((uintptr_t)x[i].data | (uintptr_t)out[i].data) % es) return refuse(DPLLM_EINVAL, "dpllm_rope: tensor %d is not aligned to its elements", i);
    all_heads += heads[i];
    if (all_heads * head_dim > (1 << 24)) return refuse(DPLLM_ESHAPE, "dpllm_rope: %lld heads of %d", (long long)all_heads, head_dim);
    a.end[i] = (int)all_heads;
    const dpllm_heads from = reached(x[i], batch, tokens, heads[i]), to = reached(out[i], batch, tokens, heads[i]);
    a.x[i] = view(from);
    a.out[i] = view(to);
    vector = vector && pieces(from, es) && pieces(to, es);
    same = same && x[i].data == out[i].data;
  }
  if (batch == 0 || tokens == 0) return DPLLM_OK;
  const int e = vector ? wide : 1;
  a.freqs = freqs_dev;
  a.positions = positions_dev;
  a.positions_stride = positions_stride;
  a.all = (int64_t)batch * tokens;
  a.tokens = tokens;
  a.heads = (int)all_heads;
  a.pairs = rotary_dim / 2;
  a.rotary = rotary_dim;
  a.turned = half ? a.pairs / e : a.pairs / (e > 1 ? e / 2 : 1);
  a.units = a.turned + (same ? 0 : (head_dim - rotary_dim) / e);
  a.scale = scale;
  a.inverse = inverse;
  const int64_t row = (int64_t)a.heads * a.units;
  // tokens enough for a workgroup's threads to have kRopeAtOnce units each on their way, but not so many that part of the chip has none
  a.at_a_time = (int)std::max<int64_t>(1, std::min<int64_t>({kRopeThreads * kRopeAtOnce / row, a.all / 512, 16}));
  a.by_tokens = Divide::by(tokens);
  a.by_units = Divide::by(a.units);
  a.by_row = Divide::by((uint32_t)row);
  a.by_pairs = Divide::by(a.pairs);
  const int64_t blocks = std::min<int64_t>((a.all + a.at_a_time - 1) / a.at_a_time, 1 << 20);
  const size_t lds = sizeof(float2) * a.at_a_time * a.pairs;
  const hipStream_t s = (hipStream_t)stream;
  if (dtype == DPLLM_F16)
    e > 1 ? launch_rope<half_t, 8>(a, half, (int)blocks, lds, s) : launch_rope<half_t, 1>(a, half, (int)blocks, lds, s);
  else if (dtype == DPLLM_BF16)
    e > 1 ? launch_rope<bfloat_t, 8>(a, half, (int)blocks, lds, s) : launch_rope<bfloat_t, 1>(a, half, (int)blocks, lds, s);
  else
    e > 1 ? launch_rope<float, 4>(a, half, (int)blocks, lds, s) : launch_rope<float, 1>(a, half, (int)blocks, lds, s);
  return launched("dpllm_rope");
}

int dpllm_cache_append(const dpllm_cache* cache, int first_layer, int n_layers, int batch, int nodes, const int32_t* lens_dev, const dpllm_heads* k_new,
                       int64_t k_layer_stride, const dpllm_heads* v_new, int64_t v_layer_stride, const int32_t* path_dev, int64_t path_stride,
                       const int32_t* count_dev, void* stream) {
  const char* who = "dpllm_cache_append";
  if (int rc = check_cache(who, cache, batch)) return rc;
  if ((!lens_dev && batch > 0) || !k_new || !v_new) return refuse(DPLLM_EINVAL, "%s: a pointer is NULL", who);
  if (first_layer < 0 || n_layers < 0 || n_layers > cache->layers - first_layer || n_layers > 65535)
    return refuse(DPLLM_ERANGE, "%s: layers %d to %lld of %d", who, first_layer, (long long)first_layer + n_layers, cache->layers);
  if (batch < 0 || nodes < 0 || nodes > (1 << 24)) return refuse(DPLLM_ESHAPE, "%s: %d sequences of %d nodes", who, batch, nodes);
  const int es = cache->dtype == DPLLM_F32 ? 4 : 2, wide = 16 / es;
  if (((uintptr_t)k_new->data | (uintptr_t)v_new->data) % es) return refuse(DPLLM_EINVAL, "%s: k_new or v_new is not aligned to its elements", who);
  if (n_layers == 0 || batch == 0 || nodes == 0) return DPLLM_OK;
  if (!k_new->data || !v_new->data) return refuse(DPLLM_EINVAL, "%s: k_new or v_new is NULL", who);
  const dpllm_cache c = reached(*cache);
  const dpllm_heads k = reached(*k_new, batch, nodes, c.heads), v = reached(*v_new, batch, nodes, c.heads);
  if (n_layers == 1) k_layer_stride = v_layer_stride = 0;
  const bool vector = c.head_dim % wide == 0 && pieces(k, es) && pieces(v, es) && (k_layer_stride | v_layer_stride) % wide == 0 &&
                      ((uintptr_t)c.k | (uintptr_t)c.v) % 16 == 0 && (c.layer_stride | c.page_stride | c.token_stride | c.head_stride) % wide == 0;
  const int e = vector ? wide : 1;
  AppendArgs a{};
  a.cache = view(c, first_layer);
  a.k = view(k);
  a.v = view(v);
  a.k_layer = k_layer_stride;
  a.v_layer = v_layer_stride;
  a.lens = lens_dev;
  a.path = path_dev;
  a.count = count_dev;
  a.path_stride = path_stride;
  a.batch = batch;
  a.tokens = nodes;
  a.head_units = cache->head_dim / e;
  a.units = a.head_units * cache->heads;
  a.by_units = Divide::by(a.units);
  a.by_head = Divide::by(a.head_units);
  // tokens for kAppendAtOnce pieces a thread: fewer leave threads without work, more leave compute units without any (11 layers of 6 sequences of 31 nodes of
  // 16 KiB: 47 us with 16 tokens to a workgroup, 14 with one)
  a.at_a_time = std::max(1, std::min(16, kAppendThreads * kAppendAtOnce / a.units));
  const dim3 grid(batch, n_layers, (nodes + a.at_a_time - 1) / a.at_a_time);
  if (grid.z > 65535) return refuse(DPLLM_ESHAPE, "%s: %d nodes", who, nodes);
  const hipStream_t s = (hipStream_t)stream;
  if (e > 1)
    hipLaunchKernelGGL(append_kernel<u32x4>, grid, dim3(kAppendThreads), 0, s, a, e);
  else if (es == 2)
    hipLaunchKernelGGL(append_kernel<uint16_t>, grid, dim3(kAppendThreads), 0, s, a, 1);
  else
    hipLaunchKernelGGL(append_kernel<uint32_t>, grid, dim3(kAppendThreads), 0, s, a, 1);
  return launched(who);
}

int dpllm_verify_workspace_bytes(int batch, int nodes, int vocabulary, int dtype, int draft, int siblings, size_t* bytes) {
  const char* who = "dpllm_verify_workspace_bytes";
  if (!bytes) return refuse(DPLLM_EINVAL, "%s: bytes is NULL", who);
  if (int rc = check_verify(who, batch, nodes, vocabulary, dtype, draft != 0, siblings)) return rc;
  *bytes = verify_space(batch, nodes, vocabulary, dtype, draft != 0, siblings).bytes;
  return DPLLM_OK;
}

int dpllm_verify(int batch, int nodes, int vocabulary, int dtype, const void* logits_dev, int64_t logits_batch_stride, int64_t logits_node_stride,
                 const void* draft_dev, int64_t draft_batch_stride, int64_t draft_node_stride, const int32_t* tokens_dev, const int32_t* parents_dev,
                 const float* uniforms_dev, const float* temperature_dev, int siblings, int32_t* count_dev, int32_t* path_dev, int32_t* words_dev, void* ws_dev,
                 size_t ws_bytes, void* stream) {
  const char* who = "dpllm_verify";
  if (int rc = check_verify(who, batch, nodes, vocabulary, dtype, draft_dev != nullptr, siblings)) return rc;
  if (batch == 0) return DPLLM_OK;
  if (!logits_dev || !tokens_dev || !uniforms_dev || !temperature_dev || !count_dev || !path_dev || !words_dev)
    return refuse(DPLLM_EINVAL, "%s: a pointer is NULL (draft_dev and parents_dev may be)", who);
  if (((uintptr_t)logits_dev | (uintptr_t)draft_dev) % (dtype == DPLLM_F32 ? 4 : 2)) return refuse(DPLLM_EINVAL, "%s: the rows are not aligned to their elements", who);
  const VerifySpace space = verify_space(batch, nodes, vocabulary, dtype, draft_dev != nullptr, siblings);
  if (!ws_dev || ws_bytes < space.bytes || (uintptr_t)ws_dev % 16)
    return refuse(DPLLM_ESTATE, "%s: needs a workspace of %zu bytes, aligned to 16", who, space.bytes);
  VerifyArgs a{};
  a.logits = (const char*)logits_dev;
  a.draft = (const char*)draft_dev;
  a.logits_batch = logits_batch_stride;
  a.logits_node = logits_node_stride;
  a.draft_batch = draft_batch_stride;
  a.draft_node = draft_node_stride;
  a.tokens = tokens_dev;
  a.parents = parents_dev;
  a.uniforms = uniforms_dev;
  a.temperature = temperature_dev;
  a.count = count_dev;
  a.path = path_dev;
  a.words = words_dev;
  a.parts = (VerifyPart*)ws_dev;
  a.rest = (double*)((char*)ws_dev + space.parts);
  a.infos = (RowInfo*)((char*)ws_dev + space.parts + space.rest);
  a.batch = batch;
  a.nodes = nodes;
  a.vocabulary = vocabulary;
  a.chunks = space.chunks;
  a.siblings = siblings;
  if (dtype == DPLLM_F16)
    launch_verify<half_t>(a, (hipStream_t)stream);
  else if (dtype == DPLLM_BF16)
    launch_verify<bfloat_t>(a, (hipStream_t)stream);
  else
    launch_verify<float>(a, (hipStream_t)stream);
  return launched(who);
}

}  // extern "C"
