"""The operators of a decode step over a quantised cache together: as examples/quantized_decode.py uses them, and as a captured step."""
import os
import sys

import pytest
import torch

import paper_2508_06041_amd as dp

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
FORMS = {"e4m3": dp.DPLLM_CACHE_E4M3, "int8": dp.DPLLM_CACHE_INT8, "int4": dp.DPLLM_CACHE_INT4}


@pytest.mark.parametrize("form", FORMS)
def test_the_example(form):
    import quantized_decode as e
    d = e.Decoder(form)
    words, kept = d.decode([5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15], 50, 0.8, top_k=40, top_p=0.9, min_p=0.01)
    assert len(words) == 50 and all(0 <= w < e.WORDS for w in words) and all(1 <= k <= 40 for k in kept)
    assert d.lens.item() == 11 + 49
    # the last token's attention over what was cached before it, in 64 bits from what the cache holds
    b, q, k, v, got = d.last
    n = d.lens.item() - 1
    keys, values = (t.double().cpu()[0] for t in dp.dpllm_quantized_read(d.cache, None, n, torch.float32, layer=b))
    keys, values = torch.cat([keys, k.double().cpu()[0]]), torch.cat([values, v.double().cpu()[0]])
    group = e.HEADS // e.KV
    keys, values = (t.repeat_interleave(group, 1) for t in (keys, values))
    scores = torch.einsum("hd,thd->ht", q.double().cpu()[0, 0], keys) * e.DIM ** -0.5
    p = torch.softmax(scores, 1)
    want = torch.einsum("ht,thd->hd", p, values)
    # scores: products of 64 terms in 32 bits, 2^-24 a step of the largest sum; weights: their rounding to float16 (the new token's), 2^-11, and at most as much again for what the scores
    # move them; then the result is rounded to float16.  All relative to the sum of the weights' products' sizes.
    size = torch.einsum("ht,thd->hd", p, values.abs())
    assert ((got.double().cpu()[0, 0] - want).abs() <= size * 2.0 ** -10 + want.abs() * 2.0 ** -11 + 2.0 ** -24).all()
    again = e.Decoder(form)
    assert again.decode([5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15], 50, 0.8, top_k=40, top_p=0.9, min_p=0.01) == (words, kept)


def test_the_best_words_are_drawn_from_alone():
    import quantized_decode as e
    words, kept = e.Decoder("int8").decode([3], 5)
    assert kept == [1] * 5 and len(words) == 5


class Step:
    """Two layers of a decode step of three sequences, without linears: everything between them, in buffers of its own."""
    LAYERS, BATCH, HEADS, KV, DIM, PAGE, PAGES = 2, 3, 8, 2, 64, 7, 9

    def __init__(self, form):
        g = torch.Generator().manual_seed(5)

        def normal(*shape):
            return torch.randn(*shape, generator=g)
        self.q, self.k, self.v = (normal(self.LAYERS, self.BATCH, 1, h, self.DIM).half().cuda() for h in (self.HEADS, self.KV, self.KV))
        self.weights = tuple((1 + 0.2 * normal(self.DIM)).cuda() for _ in range(2))
        self.freqs, self.scale = dp.dpllm_rope_frequencies(self.DIM)
        table = torch.randperm(self.BATCH * self.PAGES, generator=g).view(self.BATCH, self.PAGES).to(torch.int32).cuda()
        self.cache = dp.QuantizedCache.zeros(FORMS[form], self.LAYERS, self.BATCH * self.PAGES, self.PAGE, self.KV, self.DIM, table)
        self.lens = torch.tensor([0, 3, 13], dtype=torch.int32, device="cuda")
        self.uniforms = torch.rand(self.BATCH, generator=g).cuda()
        self.temperature, self.top_p = torch.tensor([1.0, 0.0, 0.7], device="cuda"), torch.tensor([0.9, 0.9, 1.0], device="cuda")
        self.top_k = torch.tensor([20, 0, 0], dtype=torch.int32, device="cuda")
        self.out = torch.zeros(self.LAYERS, self.BATCH, 1, self.HEADS, self.DIM, dtype=torch.float16, device="cuda")
        self.turned = torch.zeros_like(self.q), torch.zeros_like(self.k)
        self.words, self.kept = (torch.zeros(self.BATCH, dtype=torch.int32, device="cuda") for _ in range(2))

    def set(self, i):
        """What the linears would bring."""
        g = torch.Generator().manual_seed(100 + i)
        for t in (self.q, self.k, self.v):
            t.copy_(torch.randn(t.shape, generator=g).half())
        self.uniforms.copy_(torch.rand(self.BATCH, generator=g))

    def run(self):
        for i in range(self.LAYERS):
            turned = self.turned[0][i], self.turned[1][i]
            dp.dpllm_norm_rope((self.q[i], self.k[i]), self.weights, self.lens[:, None], self.freqs, out=turned, scale=self.scale)
            dp.dpllm_quantized_attention(self.cache, i, self.lens, turned[0], turned[1], self.v[i], out=self.out[i])
        dp.dpllm_quantized_append(self.cache, self.lens, self.turned[1], self.v)
        logits = self.out.sum(0).view(self.BATCH, -1) * 10
        dp.dpllm_sample(logits, self.uniforms, self.temperature, self.top_k, self.top_p, words=self.words, kept=self.kept)
        self.lens += 1

    def results(self):
        return [t.clone() for t in (*self.turned, self.out, self.words, self.kept, self.lens)]

    def held(self):
        return [t.clone() for t in (self.cache.k, self.cache.v, self.cache.k_scales, self.cache.v_scales)]


@pytest.mark.parametrize("form", FORMS)
def test_a_captured_step(form):
    """40 steps over several pages, the captured one beside the eager one: the same, bit for bit."""
    eager, captured = Step(form), Step(form)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        Step(form).run()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    for i in range(40):
        for s in (eager, captured):
            s.set(i)
        eager.run()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.results(), captured.results()):
            assert torch.equal(a, b), i
        assert (eager.words >= 0).all() and eager.kept[1] == 1
    assert eager.lens.tolist() == [40, 43, 53]
    for a, b in zip(eager.held(), captured.held()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("form", FORMS)
def test_steps_after_one_another_are_a_prompt_at_once(form):
    """Tokens that go in one by one, and all as one call: the same codes, and the same attention of the token behind them."""
    step, once = Step(form), Step(form)
    n = 20
    old = step.lens.clone()
    ks, vs = [], []
    for i in range(n):
        step.set(i)
        step.run()
        ks.append(step.turned[1].clone())
        vs.append(step.v.clone())
    dp.dpllm_quantized_append(once.cache, old, torch.cat(ks, 2), torch.cat(vs, 2))
    for a, b in zip(step.held(), once.held()):
        assert torch.equal(a, b)
    outs = [dp.dpllm_quantized_attention(s.cache, 1, old + n, step.turned[0][1]) for s in (step, once)]
    assert torch.equal(*outs)
    read = [dp.dpllm_quantized_read(s.cache, old, n, torch.float16, layer=1) for s in (step, once)]
    for a, b in zip(*read):
        assert torch.equal(a, b) and a.abs().amax() > 0


def test_a_gradient_through_the_step():
    """The norms' and rotations' gradient behind attention in torch, against differences in 64 bits of the same formula."""
    g = torch.Generator().manual_seed(9)
    q, k, v = (torch.randn(2, 6, h, 32, generator=g).cuda() for h in (4, 2, 2))
    weights = [(1 + 0.2 * torch.randn(32, generator=g)).cuda() for _ in range(2)]
    freqs, scale = dp.dpllm_rope_frequencies(32)
    positions = torch.arange(6, dtype=torch.int32, device="cuda") + 11
    leaves = [t.requires_grad_() for t in (q, k, *weights)]
    target = torch.randn(2, 6, 4, 32, generator=g)

    def attention(q, k, v):
        k, v = (t.repeat_interleave(2, 2).transpose(1, 2) for t in (k, v))
        s = q.transpose(1, 2) @ k.transpose(2, 3).contiguous() * 32 ** -0.5
        s = s.masked_fill(torch.ones(6, 6, dtype=torch.bool, device=s.device).triu(1), float("-inf"))
        return (torch.softmax(s, -1) @ v.contiguous()).transpose(1, 2)
    turned = dp.dpllm_norm_rope((q, k), weights, positions, freqs, scale=scale)
    (attention(*turned, v) * target.cuda()).sum().backward()

    def loss(q, k, wq, wk):
        def norm(x, w):
            y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
            t = positions.double().cpu()[:, None, None] * freqs.cpu()
            a, b = y[..., :16], y[..., 16:]
            return scale * torch.cat([a * torch.cos(t) - b * torch.sin(t), a * torch.sin(t) + b * torch.cos(t)], -1)
        return (attention(norm(q, wq), norm(k, wk), v.double().cpu()) * target.double()).sum()
    at = [t.detach().double().cpu() for t in leaves]
    for i, leaf in enumerate(leaves):
        d = torch.randn(leaf.shape, generator=g).double()
        h = 1e-5
        moved = (loss(*[t + h * d if j == i else t for j, t in enumerate(at)]) - loss(*[t - h * d if j == i else t for j, t in enumerate(at)])) / (2 * h)
        got = (leaf.grad.double().cpu() * d).sum()
        # 32 bits throughout: a product of sums of at most 64 terms, each good to 2^-17 of its size (as the norm's own tests say), and the difference's h^2 of a third derivative of the same order
        assert abs(got - moved) <= 2.0 ** -14 * (leaf.grad.double().cpu().abs() * d.abs()).sum(), i
