"""Calls of a step over a quantised cache at the borders of what their kernels hold at once, with nothing to do, and several at a time."""
import pytest
import torch

import paper_2508_06041_amd as dp
from test_gpu_norm_rope import check, check_gradient, plain, setup
from test_gpu_rope import normal
from test_gpu_sample import TYPES, check as check_words, numbers

pytestmark = pytest.mark.gpu
FORMS = {"e4m3": dp.DPLLM_CACHE_E4M3, "int8": dp.DPLLM_CACHE_INT8, "int4": dp.DPLLM_CACHE_INT4}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 3, 511, 512, 513, 1022, 1023, 1024, 1025, 2047, 2048, 2049, 5000])
def test_words_of_one_step(dtype, n):
    """n words within an eighth of a power of two: all different, of a few values, all the same; cuts among them by number, by sum and by both, and the words around the cut one by one."""
    v = 9000
    g = torch.Generator().manual_seed(n)
    near = torch.stack([1 + 0.04 * torch.rand(n, generator=g), 1 + 0.0625 * torch.randint(0, 2, (n,), generator=g) / 2, torch.full((n,), 1.0)])
    x = torch.full((3, v), -30.0)
    for row, words in zip(x, near):
        row[torch.randperm(v, generator=g)[:n + 1]] = torch.cat([words, torch.tensor([4.0])])
    x = x.repeat(4, 1).to(TYPES[dtype]).cuda()
    k = [0] * 3 + torch.randint(1, n + 2, (3,), generator=g).tolist() + torch.randint(max(1, n // 2), n + 2, (3,), generator=g).tolist() + [0] * 3
    p = (0.5 + 0.49 * torch.rand(12, generator=g)).tolist()
    p[3:6] = [1.0] * 3
    least = [0.0] * 9 + [0.049, 0.0495, 0.0505]      # e of the words is about e^-3 = 0.0498 and up to 4 % more
    check_words(x, numbers(12, n), [1.0] * 12, k=k, p=p, least=least)


def test_words_of_a_flat_row_at_every_number():
    """Uniform numbers all over, so that every chunk and word of what stays comes up."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn(1, 50000, generator=g).half().cuda().repeat(64, 1)
    u = ((torch.arange(64) + 0.37) / 64).tolist()
    check_words(x, u, [1.1] * 64, p=[0.93] * 64)
    check_words(x, u, [1.1] * 64, k=[1500] * 64)
    check_words(x, u, [1.1] * 64, k=[700] * 64, p=[0.8] * 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("batch,tokens,heads,kv,dim,rotary", [
    (1, 1, 1, 1, 1, 0), (2, 3, 65, 3, 2, 2), (1, 5, 300, 7, 8, 8), (1, 9, 5, 3, 16, 16), (1, 3, 33, 9, 64, 32), (2, 2, 9, 1, 513, 0), (1, 2, 2, 1, 1024, 1024), (1, 4100, 3, 1, 24, 8), (1, 2, 3, 5, 130, 126)])
def test_heads_of_all_sizes(dtype, each, batch, tokens, heads, kv, dim, rotary):
    for layout in (0, 1):
        xs, ws, pos, freqs, scale = setup(dtype, batch, tokens, heads, kv, dim, max(rotary, 2), "f32", each)
        if rotary == 0:
            pos, freqs, scale = None, None, 1.0
        grads = tuple(normal(*x.shape, dtype=x.dtype, seed=60 + i) for i, x in enumerate(xs))
        outs = dp.dpllm_norm_rope(xs, ws, pos, freqs, scale=scale, layout=layout)
        dx, dw = dp.dpllm_norm_rope_backward(xs, grads, ws, pos, freqs, scale=scale, layout=layout)
        for x, w, o, g, gx, gw in zip(xs, ws, outs, grads, dx, dw):
            check(o, *plain(x, w, pos, freqs, 1e-6, scale, layout), x.dtype)
            check_gradient((gx, gw), x, g, w, pos, freqs, 1e-6, scale, layout)


def test_nothing_to_do():
    freqs, _ = dp.dpllm_rope_frequencies(8)
    w = torch.ones(8, device="cuda"), torch.ones(3, 8, device="cuda")
    for shape in ((0, 4, 3, 8), (2, 0, 3, 8)):
        x = torch.empty(*shape, dtype=torch.bfloat16, device="cuda")
        pos = torch.empty(shape[:2], dtype=torch.int32, device="cuda")
        outs = dp.dpllm_norm_rope((x, x), w, pos, freqs)
        assert [o.shape for o in outs] == [shape] * 2
        dx, dw = dp.dpllm_norm_rope_backward((x, x), (x, x), w, pos, freqs)
        assert [d.shape for d in dx] == [shape] * 2 and all(torch.equal(d, torch.zeros_like(t)) for d, t in zip(dw, w))
    cache = dp.QuantizedCache.zeros(FORMS["int8"], 2, 4, 16, 2, 64)
    lens = torch.zeros(4, dtype=torch.int32, device="cuda")
    new = torch.empty(4, 0, 2, 64, dtype=torch.float16, device="cuda")
    dp.dpllm_quantized_append(cache, lens, new, new)
    assert dp.dpllm_quantized_attention(cache, 1, lens, torch.empty(4, 0, 8, 64, dtype=torch.float16, device="cuda")).shape == (4, 0, 8, 64)
    assert [t.shape for t in dp.dpllm_quantized_read(cache, lens, 0)] == [(4, 0, 2, 64)] * 2
    alone = dp.dpllm_quantized_attention(cache, 1, lens, torch.ones(4, 1, 8, 64, dtype=torch.float16, device="cuda"))
    assert torch.equal(alone, torch.zeros_like(alone))
    none = torch.empty(0, device="cuda")
    assert dp.dpllm_sample(torch.empty(0, 10, device="cuda"), none, none).shape == (0,)


@pytest.mark.parametrize("form", FORMS)
def test_two_streams_at_once(form):
    """The same calls on two streams, with other sizes in between so that workspaces change hands: as one after the other."""
    def run(seed, heads, n, words):
        q, k, v = (normal(3, 2, h, 128, dtype=torch.bfloat16, seed=seed + i) for i, h in enumerate((heads, 4, 4)))
        cache = dp.QuantizedCache.zeros(FORMS[form], 1, 3, n + 2, 4, 128)
        old = normal(3, n, 4, 128, dtype=torch.bfloat16, seed=seed + 3)
        zero, lens = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.full((3,), n, dtype=torch.int32, device="cuda")
        logits, u = normal(3, words, dtype=torch.float32, seed=seed + 4), torch.tensor([0.1, 0.5, 0.9], device="cuda")
        t, p = torch.ones(3, device="cuda"), torch.full((3,), 0.9, device="cuda")
        torch.cuda.synchronize()

        def step():
            dp.dpllm_quantized_append(cache, zero, old, old)
            out = dp.dpllm_quantized_attention(cache, 0, lens, q, k, v)
            turned, w = dp.dpllm_norm_rope_backward(q, out, torch.ones(128, device="cuda"))
            return out, turned, w, dp.dpllm_sample(logits, u, t, top_p=p), *dp.dpllm_quantized_read(cache, None, n)
        return step
    steps = [run(10, 16, 5000, 30000), run(20, 8, 900, 100001)]
    want = [[t.clone() for t in s()] for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(6):
        got = []
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                got.append(s())
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
