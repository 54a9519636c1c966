"""Strides of dimensions of 1 reach nothing: whatever they are, the calls around the linears give the same bits."""
import pytest
import torch

import paper_2508_06041_amd as dp
from test_gpu_tree_attention import ints, normal

pytestmark = pytest.mark.gpu


def odd(t):
    return t.as_strided(t.shape, [s if n > 1 else 12345 for n, s in zip(t.shape, t.stride())])


def tensors(*shapes, dtype=torch.float16):
    return [normal(*s, dtype=dtype, seed=i).cuda() for i, s in enumerate(shapes)]


@pytest.mark.parametrize("nodes,heads,kv,page,length", [(1, 1, 1, 16, 40), (5, 4, 1, 16, 40), (1, 8, 2, 1, 5), (3, 4, 2, 64, 64), (40, 2, 1, 16, 900)])
def test_attention(nodes, heads, kv, page, length):
    pages = -(-length // page)
    k, v, q, k_new, v_new = tensors((1, pages, page, kv, 64), (1, pages, page, kv, 64), (1, nodes, heads, 64), (1, nodes, kv, 64), (1, nodes, kv, 64))
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    want = dp.dpllm_tree_attention(dp.Cache(k, v, table), 0, ints([length]), q, k_new, v_new)
    out = odd(torch.zeros_like(q))
    got = dp.dpllm_tree_attention(dp.Cache(odd(k), odd(v), table), 0, ints([length]), odd(q), odd(k_new), odd(v_new), out=out)
    assert got is out and torch.equal(got, want) and got.count_nonzero() > 0


@pytest.mark.parametrize("batch,tokens,heads", [(1, 1, 1), (1, 7, 4), (3, 1, 2), (2, 5, 1)])
def test_rope(batch, tokens, heads):
    x, = tensors((batch, tokens, heads, 64))
    pos = torch.arange(100, 100 + tokens, dtype=torch.int32, device="cuda")
    freqs, _ = dp.dpllm_rope_frequencies(64)
    out = odd(torch.zeros_like(x))
    dp.dpllm_rope(odd(x), pos, freqs, out=out)
    assert torch.equal(out, dp.dpllm_rope(x, pos, freqs))


@pytest.mark.parametrize("layers,batch,nodes,kv,page", [(1, 1, 1, 1, 1), (1, 2, 3, 1, 16), (2, 1, 1, 4, 16)])
def test_append(layers, batch, nodes, kv, page):
    k_new, v_new = tensors((layers, batch, nodes, kv, 64), (layers, batch, nodes, kv, 64))
    table = torch.arange(4 * batch, dtype=torch.int32, device="cuda").reshape(batch, 4)
    caches = []
    for change in (lambda t: t, odd):
        k, v = (change(torch.zeros(layers, 4 * batch, page, kv, 64, dtype=torch.float16, device="cuda")) for _ in range(2))
        dp.dpllm_cache_append(dp.Cache(k, v, table), ints([1] * batch), change(k_new), change(v_new))
        caches.append((k, v))
    assert all(torch.equal(a, b) and a.count_nonzero() > 0 for a, b in zip(*caches))
