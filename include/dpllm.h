/*
 * dpllm.h — C boundary of the MI355X (gfx950) DP-LLM decode hot path.
 *
 * The library serves one multi-scale ("any-precision") weight-only-quantised model:
 * every linear keeps a parent p-bit code per weight, stored as p bitplanes, and a
 * per-row table of 2^k fp16 centroids for every k <= p, so that the k-bit model is
 * read from the top k planes only (paper Sec. 2.2: variants of 3..n bits overlaid in
 * the memory of one n-bit model).  Each linear carries a precision selector (paper
 * Sec. 3 and Sec. 5.1) that estimates the relative error ||(W_h - W_l) x|| from the
 * current input and picks h when the estimate exceeds the layer's threshold T, else l.
 *
 * Conventions
 *   - Every function returns DPLLM_OK (0) or a negative DPLLM_E* code; nothing throws
 *     or aborts.  dpllm_last_error() gives the text of the last failure on a model.
 *   - "host" / "device" on a pointer says where the memory lives.  The caller owns all
 *     device memory: the weight arenas, G, x, y, k, e, and one workspace per model
 *     (partial results of the selectors, job, task and parameter tables: some MiB, see
 *     dpllm_workspace_bytes) that it
 *     hands over with dpllm_set_workspace.  Everything is borrowed until the model is
 *     destroyed (a linear's memory: until it is loaded again).  No call allocates device
 *     memory, except dpllm_load_linear from host pointers (a staging buffer it frees
 *     before it returns).
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All work
 *     is enqueued on it; only dpllm_load_linear synchronises it.
 *   - One model may be driven from one stream at a time (the workspace is shared by
 *     the calls of a model; calls that overlap on one model race).  The calls that
 *     configure a model (load, set_selector, set_threshold, set_active_pair,
 *     set_target_entry, set_selector_input, set_workspace) take effect for the work
 *     enqueued after them and must not run while a step of the model is being captured
 *     into a graph; dpllm_set_target is the call for switching while steps are in flight.
 *   - fp16 values cross the boundary as IEEE binary16 bit patterns (uint16_t).
 *
 * Canonical host layout of a linear with `out` rows and `in` columns (in % 32 == 0):
 *   planes : uint32_t [p][out][in/32]; plane 0 = most significant bit of the p-bit
 *            code; column c is bit (c % 32) of word c / 32.
 *   luts   : luts[k - kmin] -> uint16_t [out][2^k] for k = kmin..p; the k-bit code of a
 *            weight is the top k bits of its p-bit code.
 * The library re-tiles the planes into a private, plane-separable device layout inside
 * the caller's arena; dpllm_debug_unpack returns canonical codes for checking it.
 */
#ifndef DPLLM_H
#define DPLLM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DPLLM_OK 0
#define DPLLM_EINVAL (-1) /* null pointer, bad id, bad flag, NaN threshold            */
#define DPLLM_ESHAPE (-2) /* in % 32 != 0, out < 1, batch outside [1, DPLLM_MAX_BATCH] */
#define DPLLM_ERANGE (-3) /* bitwidth outside [kmin, p] or p outside [1, 8]           */
#define DPLLM_ESTATE (-4) /* linear not loaded, selector not set, arena too small     */
#define DPLLM_EHIP (-5)   /* a HIP runtime call failed                                 */

#define DPLLM_MAX_BITS 8
#define DPLLM_MAX_BATCH 8
#define DPLLM_MAX_PAIRS 8   /* (l,h) candidate pairs kept per linear                    */
#define DPLLM_MAX_TARGETS 8 /* target precisions (sets of pairs and thresholds) resident */
#define DPLLM_MAX_RANK 1024 /* projection rank r                                        */

#define DPLLM_SEL_NONE 0   /* no estimator: always l                                     */
#define DPLLM_SEL_PROJ 1   /* random projection: e = ||G x||_2      (paper Sec. 5.1)    */
#define DPLLM_SEL_LINREG 2 /* linear regression: e = alpha ||x||_2 + beta (Sec. 5.1)    */

typedef struct dpllm_model dpllm_model; /* opaque host object */

/* Creates a model with room for n_linears linears (ids 0..n_linears-1), on the current
 * HIP device.  *out receives the handle.  Errors: EINVAL, EHIP. */
int dpllm_model_create(dpllm_model** out, int n_linears);

/* Frees the handle.  Caller-owned device memory (arenas, G, the workspace) is not
 * touched.  NULL is accepted. */
void dpllm_model_destroy(dpllm_model* m);

/* Text of the last error on m (owned by m, valid until the next failing call). */
const char* dpllm_last_error(const dpllm_model* m);

/* Bytes of device arena one linear needs (planes + tables, 256-byte aligned parts).
 * Errors: EINVAL (bytes NULL), ESHAPE, ERANGE. */
int dpllm_linear_device_bytes(int out, int in, int p, int kmin, size_t* bytes);

/* "Load a parent p-bit bitplane model with per-row LUTs for every k <= p" (Sec. 2.2).
 * Copies linear `id` from the canonical layout into dev_arena (device, caller-owned,
 * 256-byte aligned, >= dpllm_linear_device_bytes) in the private device layout.
 * src_on_device = 0: planes and every luts[i] are host pointers;
 * src_on_device = 1: they are device pointers (the array `luts` itself is always host).
 * Synchronises `stream` before returning.  Reloading an id replaces it and drops its
 * selectors.  Errors: EINVAL, ESHAPE, ERANGE, ESTATE (arena too small), EHIP. */
int dpllm_load_linear(dpllm_model* m, int id, int out, int in, int p, int kmin,
                      const uint32_t* planes, const uint16_t* const* luts, int src_on_device,
                      void* dev_arena, size_t arena_bytes, void* stream);

/* Bytes of workspace the model needs as it stands (linears loaded, pairs set): enough for every entry point and
 * every order of the linears' buffers.  Ask again after loading more linears or attaching pairs of higher rank.
 * Errors: EINVAL. */
int dpllm_workspace_bytes(const dpllm_model* m, size_t* bytes);

/* Hands the model its workspace: ws_dev (device, caller-owned, 256-byte aligned, >= dpllm_workspace_bytes), which
 * the model uses until it is destroyed or given another.  Enqueues the clearing of its target word and of what estimates
 * hand over on `stream`.
 * dpllm_estimate, dpllm_decode_step(_parts) and dpllm_set_target need a workspace; dpllm_gemv runs without one.
 * Errors: EINVAL, ESTATE (too small), EHIP. */
int dpllm_set_workspace(dpllm_model* m, void* ws_dev, size_t bytes, void* stream);

/* Attaches the precision selector of candidate pair (l, h), kmin <= l <= h <= p, to a
 * loaded linear and makes it the active pair (Sec. 3: two candidate precisions per
 * layer; Sec. 5.1: one G per pair).  kind = DPLLM_SEL_PROJ: G_dev is a device pointer
 * to fp16 [r][in] (row-major, borrowed), G = A (W_h - W_l) precomputed by the caller,
 * 1 <= r <= DPLLM_MAX_RANK.  kind = DPLLM_SEL_LINREG uses alpha, beta.  kind =
 * DPLLM_SEL_NONE needs l == h.  T may be +inf (always l) or -inf (always h), not NaN.
 * Setting an existing pair replaces it.  The pair becomes the linear's pair under target 0.
 * Errors: EINVAL, ERANGE, ESTATE. */
int dpllm_set_selector(dpllm_model* m, int id, int l, int h, int kind, const void* G_dev, int r,
                       float alpha, float beta, float T);

/* Replaces the threshold an existing pair has under target 0 and in dpllm_estimate.
 * Errors: EINVAL (NaN), ESTATE (pair not set). */
int dpllm_set_threshold(dpllm_model* m, int id, int l, int h, float T);

/* Chooses which of a linear's pairs is its pair under target 0.  Errors: ESTATE. */
int dpllm_set_active_pair(dpllm_model* m, int id, int l, int h);

/* Run-time adaptation (Sec. 2.1: the target precision changes from query to query; Algorithm 1: one threshold
 * list per target precision; Sec. 5.1: one G per candidate pair, all resident).  A model holds
 * DPLLM_MAX_TARGETS targets.  Target 0 is what dpllm_set_selector / dpllm_set_threshold / dpllm_set_active_pair
 * describe.  dpllm_set_target_entry says that under target t (1 <= t < DPLLM_MAX_TARGETS) linear id runs pair
 * (l, h), which must have been attached with dpllm_set_selector, with threshold T; a linear without an entry
 * for t runs as under target 0.  Errors: EINVAL, ESTATE (pair not set). */
int dpllm_set_target_entry(dpllm_model* m, int target, int id, int l, int h, float T);

/* Switches the whole model to `target` with one small kernel enqueued on `stream`: the steps
 * enqueued behind it (also replays of graphs captured earlier, and it can be captured itself) run every linear
 * under that target's pair and threshold.  No launch plan is rebuilt and nothing is synchronised.
 * Errors: EINVAL, ESTATE (no workspace), EHIP. */
int dpllm_set_target(dpllm_model* m, int target, void* stream);

/* Asynchronous estimation (Sec. 5.2): the selector of a layer fed by the residual stream may read the
 * previous residual vector instead of the layer's immediate input, which takes the estimate off the critical
 * path.  xsel_dev (device fp16 [in], 16-byte aligned, borrowed) replaces the input of linear id's selector in
 * dpllm_decode_step / dpllm_decode_step_parts; the GEMV still reads xs[id].  NULL restores the immediate
 * input.  The step keeps sequential semantics: a selector input written by an earlier linear of the step is
 * read after that linear has run, and when (earlier in the step) such a selector runs is the library's
 * choice.  Reloading the linear clears it.  Errors: EINVAL, ESTATE. */
int dpllm_set_selector_input(dpllm_model* m, int id, const void* xsel_dev);

/* "Estimate the relative error for (layer, x)" (Sec. 5.1) and select (Sec. 3):
 * e_dev[0] = estimate (fp32, rounded from the fp64 the decision is taken in),
 * k_dev[0] = h if estimate > T else l, for pair (l, h) of the linear and the threshold it has under target 0.
 * x_dev: device fp16 [in].  e_dev, k_dev: device.
 * Errors: EINVAL, ESTATE (pair not set, no workspace), EHIP. */
int dpllm_estimate(dpllm_model* m, int id, int l, int h, const void* x_dev, float* e_dev,
                   int32_t* k_dev, void* stream);

/* dpllm_estimate for callers that cannot allocate or hand over a workspace (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): same arguments, same result bit for bit, but the partial
 * products of the selector travel through a fixed array in the library's own device image (64 KiB per GPU, held
 * until the process ends) instead of the model's workspace.  It allocates nothing, needs no workspace, and
 * enqueues two kernels on `stream`.  Limit: projection rank r <= 256 (ERANGE beyond).  All calls on one GPU, from
 * any model or stream, share the array: calls that overlap in time on one GPU race, calls that follow one another
 * on one stream do not.  Errors: EINVAL, ERANGE, ESTATE (pair not set), EHIP. */
int dpllm_estimate_noalloc(dpllm_model* m, int id, int l, int h, const void* x_dev, float* e_dev,
                           int32_t* k_dev, void* stream);

/* "Run the GEMV at bitwidth k": y[b][o] = sum_c LUT_k[o][code_k(o,c)] * x[b][c], fp32
 * accumulation, fp16 result.  k >= 0: that bitwidth.  k < 0: the bitwidth is read on the
 * device from k_dev[0] (the hand-over from dpllm_estimate without a host round trip); a
 * value there that the linear does not serve (outside [kmin, p]) leaves y_dev untouched.  Either way, and whichever pairs
 * are attached, the same linear, B and bitwidth give the same bits.
 * x_dev: device fp16 [B][in]; y_dev: device fp16 [B][out], not overlapping x_dev;
 * 1 <= B <= DPLLM_MAX_BATCH; one bitwidth serves the whole batch.
 * Errors: EINVAL, ESHAPE, ERANGE, ESTATE, EHIP. */
int dpllm_gemv(dpllm_model* m, int id, int k, const int32_t* k_dev, const void* x_dev, void* y_dev,
               int B, void* stream);

/* "Run a whole decode step under per-layer thresholds" (Sec. 3, every linear operation
 * of every Transformer block carries a selector): for id = 0..n_linears-1 in order,
 * estimate on xs[id] with the linear's pair and threshold under the active target, then
 * the GEMV at the selected bitwidth into ys[id], batch 1, all on `stream` with no host
 * synchronisation.  xs, ys: host arrays of n_linears device pointers (fp16 [in_id], fp16
 * [out_id]; xs[id] and ys[id] must not overlap).  k_dev, e_dev: device arrays of n_linears
 * entries receiving every linear's bitwidth and estimate.  Results equal those of running
 * the linears one after another (the order of additions may differ: fp64 in the estimates,
 * fp32 in the products): consecutive linears that do not touch each other's
 * inputs and outputs share launches, dependent ones are ordered on the stream.
 * The first call, and a call after the pointers, the linears or the shapes of their pairs
 * changed, rebuilds the launch plan and copies its tables into the workspace; a call after
 * thresholds, pairs in use or target entries changed copies the parameter table.  Both are
 * asynchronous copies on `stream` (nothing is synchronised, nothing allocated) but cannot
 * be captured into a graph: ESTATE then.  Every other call only enqueues kernels.
 * A graph that holds captured steps reads these tables when it is replayed: it follows later changes of
 * thresholds, pairs in use, target entries and the target (that is the point of keeping them on the device),
 * and it must not be replayed after a call that rebuilt the launch plan for other pointers or shapes.
 * Many small linears that depend on one another run as one launch whose workgroups wait for each other's results.
 * They wait for workgroups that are running only, so the waits end whatever else the GPU does; they are bounded all the
 * same (some seconds a step).  Should one end at its bound, k_dev[0] is -1 after the step and everything else the step
 * wrote is undefined; the call itself, which only enqueues, has returned OK.
 * Errors: EINVAL, ESTATE, ESHAPE, EHIP. */
int dpllm_decode_step(dpllm_model* m, const void* const* xs, void* const* ys, int32_t* k_dev,
                      float* e_dev, void* stream);

/* The two halves of dpllm_decode_step, for callers that schedule them apart (Sec. 5.2:
 * selectors fed by an earlier activation can run ahead of the GEMVs they steer) or time
 * them apart.  parts = DPLLM_STEP_SELECT: every selector writes k_dev / e_dev.  parts =
 * DPLLM_STEP_GEMV: every GEMV runs at the bitwidth k_dev already holds (l or h of the
 * linear's active pair).  Both bits = dpllm_decode_step.  Same arguments, plan and errors. */
#define DPLLM_STEP_SELECT 1
#define DPLLM_STEP_GEMV 2
int dpllm_decode_step_parts(dpllm_model* m, const void* const* xs, void* const* ys, int32_t* k_dev,
                            float* e_dev, int parts, void* stream);

/*
 * Around the linears: what a program does with their outputs when it verifies drafted tokens (a few nodes per sequence,
 * which the small batches of dpllm_gemv serve; a draft of one token is ordinary decoding).
 *
 *   dpllm_rope            rotary positions of queries and keys, and the gradient of that
 *   dpllm_tree_attention  attention of the drafted tokens over a paged cache and over one another
 *   dpllm_verify          which drafted tokens stand against the target's probabilities, and the token after them
 *   dpllm_cache_append    the keys and values of those that stand go into the cache
 *
 * These calls need no model.  They enqueue kernels on `stream` and nothing else: nothing is synchronised, allocated or copied, and
 * all can be captured into a graph.  Lengths, page tables, masks, paths and counts are read on the device when the
 * kernels run, so replays follow them.  dpllm_call_error() gives the text of the last of them that was refused in the calling thread.
 *
 * The drafted tokens of a sequence are its nodes: node 0 is the last token that already stands (it has been fed to the
 * model together with the drafted ones), every other node has a parent with a lower number.  Node tensors are
 * [batch][nodes][heads][head_dim]; the last dimension is contiguous and the other strides are free.
 */
#define DPLLM_F16 0
#define DPLLM_BF16 1
#define DPLLM_F32 2
#define DPLLM_MAX_NODES 256    /* nodes of a tree                                        */
#define DPLLM_MAX_HEAD_DIM 1024
#define DPLLM_MAX_TENSORS 4    /* tensors of one dpllm_rope                              */

/* A device tensor [batch][tokens][heads][head_dim]; strides in elements, of head_dim 1.  The stride of a dimension of 1 may be anything (in a cache too). */
typedef struct dpllm_heads {
  void* data;
  int64_t batch_stride, token_stride, head_stride;
} dpllm_heads;

/* A paged cache of keys and values: a pool of `pages` pages of `page` tokens each, in every layer.  Token t of sequence b lies in
 * page table[b * table_stride + t / page] at place t % page; table NULL: sequence b has page b (pages_per_seq is 1).
 * A page id outside [0, pages), and a token past the sequence's pages_per_seq pages, hold nothing: they are not read, not seen, not written.
 * k and v have the same strides (elements; head_dim has 1). */
typedef struct dpllm_cache {
  void *k, *v;
  int64_t layer_stride, page_stride, token_stride, head_stride;
  const int32_t* table;
  int64_t table_stride;
  int32_t dtype, layers, pages, page, pages_per_seq, heads, head_dim;
} dpllm_cache;

/* Text of the last refusal of one of the calls from here to dpllm_sample in the calling thread (valid until the next one). */
const char* dpllm_call_error(void);

/* The angles per position that dpllm_rope takes: freqs[i], i < rotary_dim / 2 (host, radians), and *scale, what the rotated part is
 * multiplied by.  PLAIN: base^(-2i / rotary_dim).  For contexts `factor` (>= 1) times as long as the `trained` ones: LINEAR divides all by factor; NTK
 * takes base * factor^(rotary_dim / (rotary_dim - 2)); YARN goes from the plain angle to the linear one over the pairs (by number) that turn `high`
 * to `low` times over `trained` positions, and *scale = 0.1 ln(factor) + 1; BANDS goes the same way by the turns themselves
 * (at least `high`: plain, at most `low`: linear) with *scale = 1.  PLAIN, LINEAR and NTK do not use trained, low, high.
 * Errors: EINVAL, ESHAPE (rotary_dim odd or outside [2, DPLLM_MAX_HEAD_DIM]). */
#define DPLLM_ROPE_PLAIN 0
#define DPLLM_ROPE_LINEAR 1
#define DPLLM_ROPE_NTK 2
#define DPLLM_ROPE_YARN 3
#define DPLLM_ROPE_BANDS 4
int dpllm_rope_frequencies(int rotary_dim, double base, int scaling, double factor, double trained, double low, double high,
                           double* freqs, float* scale);

/* Rotary positions of up to DPLLM_MAX_TENSORS tensors (the queries and the keys, say) of the same tokens in one launch.  Pair i of a
 * head, i < rotary_dim / 2, is (i, i + rotary_dim / 2) with DPLLM_ROPE_HALF and (2i, 2i + 1) with DPLLM_ROPE_INTERLEAVED; with
 * t = position * freqs[i] it becomes scale * (a cos t - b sin t, a sin t + b cos t).  inverse != 0: -t instead, which is the
 * transpose: from the gradient of the outputs it makes the gradient of the inputs.  Elements from rotary_dim on are copied.  Angles are formed
 * in 64 bits, their sines and the products in 32, results rounded once.
 * x, out: host arrays of `tensors` views with heads[i] heads each; out[i] may be x[i] itself and must not overlap it otherwise.
 * positions_dev: int32, positions_dev[b * positions_stride + t]; positions_stride 0: the same for every sequence.  freqs_dev: fp64.
 * dtype: DPLLM_F16, DPLLM_BF16 or DPLLM_F32.  batch or tokens 0: nothing to do.
 * Errors: EINVAL, ESHAPE, EHIP. */
#define DPLLM_ROPE_HALF 0
#define DPLLM_ROPE_INTERLEAVED 1
int dpllm_rope(const dpllm_heads* x, const dpllm_heads* out, const int* heads, int tensors, int batch, int tokens, int head_dim,
               int dtype, int rotary_dim, int layout, const double* freqs_dev, float scale, const int32_t* positions_dev,
               int64_t positions_stride, int inverse, void* stream);

/* Attention of the nodes over what the cache holds and over one another: for every node i and query head h of sequence b,
 * out = softmax_t(scale q . k_t) v over the tokens t < lens[b] of the cache (kv head h / (heads / cache->heads)) and those nodes j whose bit is set in
 * row i of the mask: bit j % 64 of word mask[b * mask_stride + i * ceil(nodes / 64) + j / 64]; mask_stride 0: one mask for all sequences.  A node sees itself only if
 * its own bit says so.  mask_dev NULL: the nodes are a chain, i sees j <= i.  k_new and v_new NULL: the cache only.  Nothing that is not seen is
 * read as a number: infinities and NaN there change nothing.  A row that sees nothing (or scores of minus infinity only) is zero, its lse minus infinity;
 * one that sees a score of NaN or plus infinity is NaN, and so is its lse.  lens: negative is 0, and no
 * more than the sequence's pages hold.  max_len: how long the longest is expected to be; it sets how the work is split, not the result.
 * q, out: [batch][nodes][heads][head_dim]; k_new, v_new: [batch][nodes][cache->heads][head_dim]; all of the cache's type, DPLLM_F16 or DPLLM_BF16,
 * 16-byte aligned, strides multiples of 8 elements.  head_dim 64, 96, 128 or 256; heads a multiple of cache->heads; nodes up to DPLLM_MAX_NODES.
 * lse_dev: float [batch][nodes][heads], the logarithm of the sum of exp(scale q . k_t), or NULL.  Scores, maxima and sums are kept in 32 bits, the weights
 * are rounded to the type of v for the product with it.  ws_dev: 16-byte aligned, of at least dpllm_tree_attention_workspace_bytes for the same sizes (0:
 * NULL is accepted), used until the call's kernels have run.  out must not overlap the inputs.  The same call gives the same bits.
 * Errors: EINVAL, ESHAPE, ERANGE (layer), ESTATE (workspace), EHIP. */
int dpllm_tree_attention_workspace_bytes(int batch, int nodes, int heads, int kv_heads, int head_dim, int max_len, size_t* bytes);
int dpllm_tree_attention(const dpllm_cache* cache, int layer, int batch, int nodes, int heads, const int32_t* lens_dev, int max_len,
                         const dpllm_heads* q, const dpllm_heads* k_new, const dpllm_heads* v_new, const uint64_t* mask_dev,
                         int64_t mask_stride, float scale, const dpllm_heads* out, float* lse_dev, void* ws_dev, size_t ws_bytes,
                         void* stream);

/* Which drafted tokens stand, and the token behind them.  Row i of `logits` is the target's answer behind node i, p_i = softmax(logits_i / temperature[b]);
 * row i of `draft` the draft's, q_i, from which the tokens of i's children were drawn, each by itself.  From the root (node 0) on, the children of a node are
 * asked in the order of their numbers: child c stands if uniforms[c] q(c) < r(c), where r is p at first and norm(max(r - q, 0)) behind every child that
 * did not stand (r stays where nothing is left; a word of which no more than 4e-13 is left has nothing, as equal rows may come to that).  With draft_dev NULL the children were named, not drawn: c stands if uniforms[c] < r(c), and a
 * child that does not leaves r (unless it is all there is, to 4e-13).  The first child that stands is the next node; where none does, the token behind is drawn from r: the first word whose running sum of r exceeds uniforms[0] times
 * the whole, words of less than 1e-280 left out.  Tokens so chosen are distributed as if drawn from the target.  temperature[b] 0 (or less, or NaN): a child stands if it is the word with
 * the largest logit, the lowest such word where several are, and that word is the token behind; the draft rows are not read.
 * logits, draft: dtype [batch][nodes][vocabulary], the words contiguous, strides in elements.  tokens: int32 [batch][nodes] (that of node 0 is not read); a token outside the
 * vocabulary never stands.  parents: int32 [batch][nodes]; a node whose parent is not a lower node is nobody's child; NULL: a chain.  uniforms: float
 * [batch][nodes] in [0, 1).  temperature: float [batch].  Logits of minus infinity and NaN have probability 0; where one is plus infinity, only such have any.
 * siblings (with draft rows only): the most children that a node has; a call makes that many passes over the rows whose children are refused, two launches each.  Where a node has
 * more, those beyond that did not stand leave r as it was and the children behind them are not asked.
 * count [batch]: how many nodes stand, the root among them, which is also how many tokens there are in words.  path [batch][nodes]: those nodes.  words [batch][nodes]:
 * the tokens of the drafted ones among them, then the token behind (-1 where the last row has no finite logit).  The rest of both is -1.  path and count are
 * what dpllm_cache_append takes.  Logits are widened and everything is computed in 64 bits, so the answers do not depend on the order of additions but for ties to 1e-13.
 * ws_dev: 16-byte aligned, of dpllm_verify_workspace_bytes, used until the call's kernels have run.  Errors: EINVAL, ESHAPE, ESTATE (workspace), EHIP. */
int dpllm_verify_workspace_bytes(int batch, int nodes, int vocabulary, int dtype, int draft, int siblings, size_t* bytes);
int dpllm_verify(int batch, int nodes, int vocabulary, int dtype, const void* logits_dev, int64_t logits_batch_stride,
                 int64_t logits_node_stride, const void* draft_dev, int64_t draft_batch_stride, int64_t draft_node_stride,
                 const int32_t* tokens_dev, const int32_t* parents_dev, const float* uniforms_dev, const float* temperature_dev,
                 int siblings, int32_t* count_dev, int32_t* path_dev, int32_t* words_dev, void* ws_dev, size_t ws_bytes, void* stream);

/* Puts keys and values of some nodes behind what the cache holds, for n_layers layers from first_layer on: node path[b][i] of sequence b goes to token
 * lens[b] + i, i < count[b] (rows of path are path_stride entries apart and hold `nodes`).  path_dev NULL: nodes in their order; count_dev NULL: all nodes.  Entries of path outside [0, nodes), tokens without a
 * page and sequences with a negative length are left out; counts above nodes are taken as nodes.  lens is not changed (add the counts
 * behind the call).  k_new, v_new: views of one layer's [batch][nodes][heads][head_dim] with the cache's type, layers k_layer_stride and v_layer_stride
 * elements apart; they must not overlap the cache.  Slots that two sequences share take either's values.
 * Errors: EINVAL, ESHAPE, ERANGE (layers), EHIP. */
int dpllm_cache_append(const dpllm_cache* cache, int first_layer, int n_layers, int batch, int nodes, const int32_t* lens_dev,
                       const dpllm_heads* k_new, int64_t k_layer_stride, const dpllm_heads* v_new, int64_t v_layer_stride,
                       const int32_t* path_dev, int64_t path_stride, const int32_t* count_dev, void* stream);

/*
 * A cache in 8 or 4 bits, and what else a decode step does between its linears.  On the same terms as the calls above.
 *
 *   dpllm_norm_rope            norms of queries and keys for each head and their rotary positions in one pass, and the gradient of that
 *   dpllm_quantized_append     keys and values are quantised as they go into the cache
 *   dpllm_quantized_read       and come back
 *   dpllm_quantized_attention  attention of new tokens over such a cache and over one another
 *   dpllm_sample               the next token: temperature, top-k, top-p and min-p
 */

/* Norms of the heads of up to DPLLM_MAX_TENSORS tensors (the queries and the keys, say) of the same tokens, with a learned weight each, and their rotary positions:
 * n = x / sqrt(mean of x^2 over the head + eps), out = the rotation of dpllm_rope (layout, freqs_dev, scale, positions) of weight * n.  rotary_dim 0: no rotation; freqs_dev and
 * positions_dev may be NULL.  weights: host array of `tensors` device pointers (or NULL: all are 1; so is one that is NULL), each [head_dim] for all heads where
 * weight_strides[i] is 0, else of head h from weight_strides[i] * h on, of weight_dtype.  x, out, heads, dtype, positions: as for dpllm_rope; out[i] may be x[i]
 * itself and must not overlap it otherwise.  Sums and products are in 32 bits, results are rounded once.
 * backward: from the gradients of the outputs, grads[i], it makes those of the inputs, grad_x[i] (which may be grads[i] or x[i] itself), and of the weights, grad_weights[i] (NULL: none is
 * wanted; as NULL is for the array), which are laid out as the weights and summed over tokens, and over heads that share one, in 32 bits, in the same order every time.  ws_dev: 16-byte aligned, of
 * dpllm_norm_rope_backward_workspace_bytes for the same sizes (0: NULL is accepted), used until the call's kernels have run.
 * batch or tokens 0: nothing to do but to clear the gradients of weights.  Errors: EINVAL, ESHAPE, ESTATE (workspace), EHIP. */
int dpllm_norm_rope(const dpllm_heads* x, const dpllm_heads* out, const int* heads, const void* const* weights, const int64_t* weight_strides, int weight_dtype,
                    float eps, int tensors, int batch, int tokens, int head_dim, int dtype, int rotary_dim, int layout, const double* freqs_dev, float scale,
                    const int32_t* positions_dev, int64_t positions_stride, void* stream);
int dpllm_norm_rope_backward_workspace_bytes(const int* heads, const int64_t* weight_strides, int tensors, int batch, int tokens, int head_dim, size_t* bytes);
int dpllm_norm_rope_backward(const dpllm_heads* x, const dpllm_heads* grads, const dpllm_heads* grad_x, const int* heads, const void* const* weights,
                             void* const* grad_weights, const int64_t* weight_strides, int weight_dtype, float eps, int tensors, int batch, int tokens, int head_dim, int dtype,
                             int rotary_dim, int layout, const double* freqs_dev, float scale, const int32_t* positions_dev, int64_t positions_stride, void* ws_dev,
                             size_t ws_bytes, void* stream);

/* A paged cache as dpllm_cache, whose keys and values are codes with one 32-bit word for each token and head (k_scales, v_scales):
 *   E4M3  a byte each, OCP e4m3; the word is a float, the smallest power of two with which the largest size of the head is at most 448
 *   INT8  a byte each, -127 ... 127, round(127 x / the largest size); the word is a float, the largest size / 127
 *   INT4  half a byte each, element 2i in the lower half of byte i: bit 3 the sign, m below, for offset +- scale (m + 1/2).  The word is two bfloat16: the scale in the lower
 *         half, the offset in the upper.  offset = (lowest + highest) / 2; scale = an eighth of the larger distance of those from it, rounded up, or 0 where they are equal;
 *         a value is at floor((x - offset) / scale), within -8 ... 7.  (Where offset or scale are past the largest bfloat16, which only floats next to the largest come to, the head is held as NaN.)
 * Sizes (and distances) below 2^-100 that are not 0 count as 2^-100.  A head with a value that is no finite number is held as NaN.
 * Strides of codes are in bytes, those of scales in words, the same for keys and values; the codes of a head lie side by side. */
#define DPLLM_CACHE_E4M3 1
#define DPLLM_CACHE_INT8 2
#define DPLLM_CACHE_INT4 3
typedef struct dpllm_quantized_cache {
  void *k, *v, *k_scales, *v_scales;
  int64_t layer_stride, page_stride, token_stride, head_stride;
  int64_t scale_layer_stride, scale_page_stride, scale_token_stride, scale_head_stride;
  const int32_t* table;
  int64_t table_stride;
  int32_t format, layers, pages, page, pages_per_seq, heads, head_dim;
} dpllm_quantized_cache;

/* dpllm_cache_append into such a cache; k_new and v_new are of `dtype` (DPLLM_F16, DPLLM_BF16 or DPLLM_F32).  A slot that two sequences share may end with one's codes
 * and the other's scale: sequences may share pages only where none of them is written.  head_dim up to DPLLM_MAX_HEAD_DIM, even for INT4.
 * Errors: EINVAL, ESHAPE, ERANGE (layers), EHIP. */
int dpllm_quantized_append(const dpllm_quantized_cache* cache, int first_layer, int n_layers, int batch, int nodes, const int32_t* lens_dev, int dtype,
                           const dpllm_heads* k_new, int64_t k_layer_stride, const dpllm_heads* v_new, int64_t v_layer_stride, const int32_t* path_dev,
                           int64_t path_stride, const int32_t* count_dev, void* stream);

/* What the cache holds of tokens first[b] ... + tokens - 1 of every sequence, for n_layers layers from first_layer on, into k_out and v_out: [layers][batch][tokens][heads][head_dim]
 * of `dtype`, layers k_layer_stride and v_layer_stride elements apart.  first_dev NULL: from token 0 on.  count_dev NULL: all of them, else those from count[b] on are written as zeros, as are
 * tokens that no page holds (those in front of token 0 among them).  Values are products (and sums), formed in 32 bits or exactly and rounded to dtype.
 * Errors: EINVAL, ESHAPE, ERANGE (layers), EHIP. */
int dpllm_quantized_read(const dpllm_quantized_cache* cache, int first_layer, int n_layers, int batch, int tokens, const int32_t* first_dev, const int32_t* count_dev,
                         int dtype, const dpllm_heads* k_out, int64_t k_layer_stride, const dpllm_heads* v_out, int64_t v_layer_stride, void* stream);

/* dpllm_tree_attention over such a cache: the same arguments and rules, with `dtype` (DPLLM_F16 or DPLLM_BF16) the type of q, k_new, v_new and out, which are not quantised.  The
 * cached tokens count as what their codes and scales stand for, unrounded; the products of their weights and the scales of their values are rounded to 16 bits for the value product, whatever their size, and
 * the weights of the new tokens likewise (to 22 bits where the type is float16).  Codes and their strides are aligned to 16 bytes.  A head that holds NaN makes NaN of the rows that see it.
 * Errors: EINVAL, ESHAPE, ERANGE (layer), ESTATE (workspace), EHIP. */
int dpllm_quantized_attention_workspace_bytes(int batch, int nodes, int heads, int kv_heads, int head_dim, int max_len, size_t* bytes);
int dpllm_quantized_attention(const dpllm_quantized_cache* cache, int layer, int batch, int nodes, int heads, int dtype, const int32_t* lens_dev, int max_len,
                              const dpllm_heads* q, const dpllm_heads* k_new, const dpllm_heads* v_new, const uint64_t* mask_dev, int64_t mask_stride, float scale,
                              const dpllm_heads* out, float* lse_dev, void* ws_dev, size_t ws_bytes, void* stream);

/* A word for every row of logits [rows][vocabulary] (dtype, the words contiguous, rows `stride` elements apart) by a given uniform number.  Words are ordered by their logits, the largest
 * first, equal ones by their numbers, with weights e = exp((logit - largest) / temperature[row]); those of less than 2^-64 are left out.  Of the others stay
 *   the first top_k[row] (0 or less: all);
 *   of these each in front of which less than top_p[row] of their sum lies (1 or more, or NaN: all; the first always stays);
 *   of these each with e at least min_p[row] (0 or less, or NaN: all; the first always stays).
 * words[row] is the first of them, by number, whose running sum (by number) exceeds uniforms[row] times their whole: what dpllm_verify draws behind a lone node
 * where nothing is filtered.  kept[row], if kept_dev is not NULL: how many stayed.  temperature 0 (or less, or NaN): the largest logit, the lowest such word where several are.  Logits of minus infinity and NaN
 * never stay; where one is plus infinity only such do, with equal weights.  A row without a word to draw gives -1 (and keeps 0).  top_k, top_p, min_p, temperature, uniforms: [rows] on the
 * device; the first three may be NULL.  Everything is computed in 64 bits, in an order that does not change.  ws_dev: 16-byte aligned, of
 * dpllm_sample_workspace_bytes, used until the call's kernels have run.  Errors: EINVAL, ESHAPE, ESTATE (workspace), EHIP. */
int dpllm_sample_workspace_bytes(int rows, int vocabulary, int dtype, size_t* bytes);
int dpllm_sample(int rows, int vocabulary, int dtype, const void* logits_dev, int64_t stride, const float* uniforms_dev, const float* temperature_dev,
                 const int32_t* top_k_dev, const float* top_p_dev, const float* min_p_dev, int32_t* words_dev, int32_t* kept_dev, void* ws_dev, size_t ws_bytes,
                 void* stream);

/* Parity aid: writes the canonical k-bit codes of linear `id`, uint8 [out][in], read back
 * from the private device layout, to idx_dev (device).  Errors: EINVAL, ERANGE, ESTATE, EHIP. */
int dpllm_debug_unpack(dpllm_model* m, int id, int k, uint8_t* idx_dev, void* stream);

/* Parity aid (host only, touches no device): where the private device layout keeps the plane-`plane` bit of the
 * weight (row, col) of a linear of this shape: *byte_offset from the start of the arena (a multiple of 4: the
 * 32-bit word), *bit inside that word.  Errors: EINVAL, ESHAPE, ERANGE. */
int dpllm_debug_locate(int out, int in, int p, int kmin, int plane, int row, int col, size_t* byte_offset, int* bit);

/* Parity aid: how often a workgroup of a step looks for products of its linear's selector that other workgroups of the
 * launch deliver, before it computes them all itself (64 looks of about a microsecond unless set; dpllm_estimate then
 * looks a million times).  0: it looks once; -1: it looks once and, in a step, nobody delivers any.  The results are the same bits.  (A step that is one launch in all does not
 * ask: see dpllm_debug_set_one_launch.)  Errors: EINVAL. */
int dpllm_debug_set_polls(dpllm_model* m, int polls);

/* Parity aid: whether a step of dependent linears is one launch whose workgroups hand the results over themselves.
 * 0 (unless set): where that is faster, by the linears' shapes and the ranks of their pairs; 1: wherever the buffers allow
 * it; -1: never.  seats > 0: the first linears of such a launch are dealt out to at most so many workgroups, and the others
 * join later, as they do where the chip is busy with other work (0, unless set: no bound).  The next step rebuilds the launch
 * plan.  mode changes the order of additions, seats no bit of the results.  Errors: EINVAL. */
int dpllm_debug_set_one_launch(dpllm_model* m, int mode, int seats);

/* Parity aid: how many kernels the model's last step was made of (one launch for all linears: 2, one of them clears
 * what the other hands over).  Errors: EINVAL. */
int dpllm_debug_step_launches(const dpllm_model* m, int* launches);

/* Measurement aid: a plain 128-bit copy kernel, bytes % 16 == 0, both pointers device and 16-byte
 * aligned.  Its known traffic (bytes read + bytes written) scales the HBM byte counters that the
 * profiles report for the GEMV.  Errors: EINVAL, EHIP. */
int dpllm_debug_copy(void* dst_dev, const void* src_dev, size_t bytes, void* stream);

/* Measurement aid: a plain 128-bit non-temporal streaming read of `bytes` (bytes % 16 == 0, pointers device and
 * 16-byte aligned; sink_dev: 16 writable bytes, practically never written).  Its rate over >= 1 GiB is the
 * measured HBM read ceiling the GEMV's rate is reported against.  Errors: EINVAL, EHIP. */
int dpllm_debug_read(const void* src_dev, size_t bytes, void* sink_dev, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DPLLM_H */
