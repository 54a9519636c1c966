"""Words drawn with temperature, top-k, top-p and min-p from given uniform numbers, against a sort in 64 bits on the CPU."""
import math

import numpy as np
import pytest
import torch

import paper_2508_06041_amd as dp

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def plain(x, u, temperature, k, p, least):
    """The word and how many stayed, of one row (numpy, 64 bits)."""
    x = np.where(np.isnan(x), -np.inf, x)
    if x.size == 0 or x.max() == -np.inf:
        return -1, 0
    if not temperature > 0:
        return int(x.argmax()), 1
    order = np.lexsort((np.arange(x.size), -x))
    top = x.max()
    with np.errstate(invalid="ignore", over="ignore"):
        e = np.exp(np.where(x == top, 0.0, (x - top) / temperature))
    e = np.where(np.isneginf(x), 0.0, e)      # also where the temperature is infinite
    e = np.where(np.isnan(e), 0.0, e)[order]
    n = int((e >= 2.0 ** -64).sum())
    if k is not None and k > 0:
        n = min(n, k)
    front = np.concatenate([[0.0], np.cumsum(e[:n])])
    if p is not None and p < 1:
        n = max(1, int((front[:n] < p * front[n]).sum()))
    if least is not None and least > 0:
        n = max(1, int((e[:n] >= least).sum())) if least <= 1 else 1
    kept = order[:n]
    w = np.zeros(x.size)
    w[kept] = e[:n]
    run = np.cumsum(w)
    return int(np.argmax(run > u * run[-1])), n


def check(logits, u, temperature, k=None, p=None, least=None):
    def on(v, dtype):
        return None if v is None else torch.tensor(v, dtype=dtype, device="cuda")
    n = logits.shape[0]
    kept = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    got = dp.dpllm_sample(logits, on(u, torch.float32), on(temperature, torch.float32), top_k=on(k, torch.int32), top_p=on(p, torch.float32), min_p=on(least, torch.float32),
                          kept=kept)
    x = logits.double().cpu().numpy()

    def row(v, i):
        return None if v is None else float(np.float32(v[i])) if isinstance(v[i], float) else v[i]
    want = [plain(x[i], row(u, i), row(temperature, i), row(k, i), row(p, i), row(least, i)) for i in range(n)]
    assert kept.tolist() == [m for _, m in want]
    assert got.tolist() == [w for w, _ in want]
    return got


def rows(n, v, dtype, seed, boost=9.0, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, v, generator=g) * spread
    x.scatter_add_(1, torch.randint(0, v, (n, 8), generator=g), torch.full((n, 8), boost))
    return x.to(TYPES[dtype]).cuda()


def numbers(n, seed):
    return torch.rand(n, generator=torch.Generator().manual_seed(seed)).tolist()


SETTINGS = [dict(), dict(k=[40]), dict(k=[1]), dict(k=[1500]), dict(p=[0.9]), dict(p=[0.3]), dict(p=[0.999]), dict(least=[0.05]), dict(least=[1e-6]), dict(k=[60], p=[0.9], least=[0.02]),
            dict(k=[3000], p=[0.99]), dict(k=[20000], p=[0.9999], least=[1e-9]), dict(k=[0], p=[1.0], least=[0.0]), dict(k=[10 ** 9], p=[1.5], least=[-1.0]), dict(p=[0.0]), dict(p=[-1.0], k=[5]),
            dict(p=[math.nan], least=[math.nan]), dict(least=[1.0]), dict(least=[2.0]), dict(k=[-3], p=[1e-9])]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v", [1, 2, 7, 64, 1000, 4097, 32000, 128256])
def test_every_filter(dtype, v):
    """Peaked and flat rows; with a small vocabulary a word stands above nothing."""
    for boost, seed in ((9.0, 1), (14.0, 2), (0.0, 3)):
        for i, s in enumerate(SETTINGS):
            n = 4
            check(rows(n, v, dtype, seed * 100 + i, boost), numbers(n, seed * 1000 + i), [1.0, 0.7, 1.3, 0.25], **{name: value * n for name, value in s.items()})


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_with_their_own_settings(dtype):
    n = 48
    g = torch.Generator().manual_seed(4)
    k = torch.randint(-1, 200, (n,), generator=g).tolist()
    p = (torch.rand(n, generator=g) * 1.2).tolist()
    least = (torch.rand(n, generator=g) * 0.2 - 0.1).tolist()
    temperature = (torch.rand(n, generator=g) * 2 - 0.3).tolist()
    check(rows(n, 50257, dtype, 5, 12.0), numbers(n, 6), temperature, k, p, least)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v", [3000, 100001])
def test_equal_words(dtype, v):
    """All the same; a few values with many words each; cuts in the middle of them, which go by number."""
    flat = torch.full((6, v), 1.5, dtype=TYPES[dtype], device="cuda")
    check(flat, numbers(6, 1), [1.0] * 6, k=[0, 1, 1000, v // 2, v - 1, 0], p=[1.0, 1.0, 0.5, 1.0, 0.25, 0.77])
    x = torch.randint(0, 4, (8, v), generator=torch.Generator().manual_seed(2)).to(TYPES[dtype]).cuda()
    check(x, numbers(8, 3), [1.0, 0.5, 1.0, 2.0, 1.0, 1.0, 1.0, 1.0], k=[0, v // 8, v // 3, v // 2, v * 3 // 4, 10, 0, v // 2], p=[0.3, 1.0, 0.9, 0.5, 0.99, 1.0, 0.95, 0.9999],
          least=[0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.06, 0.2])


@pytest.mark.parametrize("dtype", TYPES)
def test_many_words_in_one_step(dtype):
    """More words within an eighth of a power of two than are sorted at once, different ones and not."""
    g = torch.Generator().manual_seed(9)
    x = (torch.rand(6, 60000, generator=g) * 0.08).to(TYPES[dtype]).cuda()
    check(x, numbers(6, 10), [1.0, 1.0, 0.9, 1.1, 1.0, 1.0], k=[0, 30000, 5000, 59999, 41000, 2049], p=[0.5, 1.0, 0.9, 0.33, 0.999, 0.99])


@pytest.mark.parametrize("dtype", TYPES)
def test_numbers_that_are_none(dtype):
    t = TYPES[dtype]
    x = rows(8, 9000, dtype, 11)
    x[0, ::2] = math.nan
    x[1, :] = -math.inf
    x[2, :] = math.nan
    x[3, 100:200] = math.inf
    x[4, 5:] = -math.inf
    x[5, 7] = torch.finfo(t).max
    x[6, :] = -torch.finfo(t).max
    x[7, 8999] = math.inf
    for k, p, least in ((None, None, None), ([50] * 8, None, None), (None, [0.9] * 8, None), ([7] * 8, [0.5] * 8, [0.1] * 8)):
        check(x, numbers(8, 12), [1.0] * 8, k, p, least)
    check(x, numbers(8, 13), [0.0] * 8)


def test_temperatures_and_uniforms():
    x = rows(10, 5000, "f32", 14)
    check(x, numbers(10, 15), [0.0, -1.0, math.nan, 1e-30, 1e-3, 1e30, math.inf, 1e-42, 100.0, 0.01], k=[0, 0, 0, 0, 3, 0, 0, 2, 4000, 0], p=[0.9] * 5 + [1.0] * 5)
    check(x, [0.0, 1 - 2.0 ** -24] * 5, [1.0] * 10, k=[0] * 5 + [20] * 5)
    one = rows(1, 100, "f32", 16).expand(256, 100)                     # one row for all (no stride), every part of its words
    check(one, [i / 256 for i in range(256)], [1.0] * 256, k=[30] * 256)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift,gap", [(0, 3), (1, 0), (3, 5)])
def test_rows_at_any_address(dtype, shift, gap):
    v, n = 8200, 5
    space = rows(1, shift + n * (v + gap), dtype, 17)[0]
    x = space[shift:shift + n * (v + gap)].view(n, v + gap)[:, :v]
    check(x, numbers(n, 18), [1.0] * n, k=[0, 50, 0, 4000, 8], p=[1.0, 1.0, 0.9, 0.97, 0.5])


def test_as_a_lone_node_is_verified():
    """Without a filter the draw is that of dpllm_verify behind a node without children."""
    x = rows(16, 30000, "bf16", 19)
    u, t = torch.tensor(numbers(16, 20), device="cuda"), torch.full((16,), 0.8, device="cuda")
    _, _, words = dp.dpllm_verify(x[:, None], torch.zeros(16, 1, dtype=torch.int32, device="cuda"), u[:, None].contiguous(), t)
    assert torch.equal(dp.dpllm_sample(x, u, t), words[:, 0])


def test_no_rows_and_given_outputs():
    x = rows(3, 500, "f16", 21)
    u, t = torch.tensor(numbers(3, 22), device="cuda"), torch.ones(3, device="cuda")
    want = dp.dpllm_sample(x, u, t)
    words = torch.empty(3, dtype=torch.int32, device="cuda")
    space = torch.empty(dp.dpllm_sample_workspace_bytes(3, 500, dp.DPLLM_F16), dtype=torch.uint8, device="cuda")
    assert dp.dpllm_sample(x, u, t, words=words, workspace=space) is words and torch.equal(words, want)
    assert dp.dpllm_sample(x[:0], u[:0], t[:0]).shape == (0,)


def test_graphs_that_share_a_workspace():
    x = rows(5, 40000, "bf16", 23)
    u, t = torch.tensor(numbers(5, 24), device="cuda"), torch.ones(5, device="cuda")
    k, p = torch.tensor([0, 20, 0, 5000, 7], dtype=torch.int32, device="cuda"), torch.tensor([1.0, 0.9, 0.95, 0.99, 1.0], device="cuda")
    space = torch.empty(dp.dpllm_sample_workspace_bytes(5, 40000, dp.DPLLM_BF16), dtype=torch.uint8, device="cuda")
    words = [torch.zeros(5, dtype=torch.int32, device="cuda") for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for i in range(2):
        def step():
            dp.dpllm_sample(x, u, t, top_k=k if i else None, top_p=p, words=words[i], workspace=space)
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for turn in range(4):
        x.copy_(rows(5, 40000, "bf16", 30 + turn))
        u.copy_(torch.tensor(numbers(5, 40 + turn)))
        t.fill_([1.0, 0.5, 0.0, 2.0][turn])
        k.add_(3)
        want = [dp.dpllm_sample(x, u, t, top_k=k if i else None, top_p=p) for i in range(2)]
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(words, want))
