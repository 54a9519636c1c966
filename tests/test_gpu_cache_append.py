"""Keys and values of the tokens that stand, into the pages of the cache: bit for bit against a loop."""
import pytest
import torch

import paper_2508_06041_amd as dp

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def normal(*shape, dtype, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def plain(k, v, table, lens, k_new, v_new, path, count, layer):
    """All on the CPU; k, v: [layers][pages][page][heads][d]."""
    page = k.shape[2]
    n = k_new.shape[2]
    for b, first in enumerate(lens):
        for i in range(n if count is None else min(count[b], n)):
            src = i if path is None else path[b][i]
            at = first + i
            if first < 0 or not 0 <= src < n or at // page >= len(table[b]) or not 0 <= table[b][at // page] < k.shape[1]:
                continue
            for l in range(k_new.shape[0]):
                k[layer + l, table[b][at // page], at % page] = k_new[l, b, src]
                v[layer + l, table[b][at // page], at % page] = v_new[l, b, src]


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layers,layer,batch,nodes,heads,dim,page,each", [
    (1, 0, 1, 1, 1, 1, 1, 3), (3, 0, 2, 5, 2, 64, 16, 2), (4, 1, 3, 9, 8, 128, 1, 40), (2, 1, 2, 40, 3, 33, 7, 9), (2, 0, 5, 17, 1, 96, 32, 3)])
@pytest.mark.parametrize("paths", [False, True])
def test_against_a_loop(dtype, layers, layer, batch, nodes, heads, dim, page, each, paths):
    g = torch.Generator().manual_seed(1)
    t, pages = TYPES[dtype], batch * each + 2
    k, v = normal(layers, pages, page, heads, dim, dtype=t, seed=2), normal(layers, pages, page, heads, dim, dtype=t, seed=3)
    k_new, v_new = normal(layers - layer, batch, nodes, heads, dim, dtype=t, seed=4), normal(layers - layer, batch, nodes, heads, dim, dtype=t, seed=5)
    table = (torch.randperm(pages, generator=g)[:batch * each]).reshape(batch, each).tolist()
    table[-1][-1] = -1                       # no page there
    if batch > 1:
        table[0][0] = pages                  # nor there
    lens = torch.randint(0, each * page, (batch,), generator=g).tolist()      # some run over the end
    if batch > 2:
        lens[1] = -1
    path = [torch.randint(-1, nodes + 1, (nodes,), generator=g).tolist() for _ in range(batch)] if paths else None
    count = torch.randint(0, nodes + 3, (batch,), generator=g).tolist() if paths else None
    dk, dv = k.cuda(), v.cuda()
    for _ in range(2):                       # a second time changes nothing
        dp.dpllm_cache_append(dp.Cache(dk, dv, ints(table)), ints(lens), k_new.cuda(), v_new.cuda(), path=ints(path), count=ints(count), layer=layer)
        plain(k, v, table, lens, k_new, v_new, path, count, layer)
        assert torch.equal(dk.cpu().view(torch.uint8), k.view(torch.uint8)) and torch.equal(dv.cpu().view(torch.uint8), v.view(torch.uint8))


def test_layouts_and_no_table():
    """Pages that hold head after head, nodes as slices of a projection and at odd addresses, one stretch per sequence."""
    for shift in (0, 1):
        pool = normal(2, 2 * 3 * 50 * 64 * 2 + 8, dtype=torch.float16, seed=6).cuda()
        k, v = (pool[i, shift:shift + 2 * 3 * 50 * 64].view(1, 3, 2, 50, 64).transpose(2, 3) for i in range(2))     # [1][3][50][2][64]
        qkv = normal(3, 4, 8, 64, dtype=torch.float16, seed=7).cuda()
        wk, wv = k.cpu().clone(), v.cpu().clone()
        dp.dpllm_cache_append(dp.Cache(k, v), ints([0, 46, 49]), qkv[:, :, 4:6], qkv[:, :, 6:])
        plain(wk, wv, [[0], [1], [2]], [0, 46, 49], qkv[None, :, :, 4:6].cpu(), qkv[None, :, :, 6:].cpu(), None, None, 0)
        assert torch.equal(k.cpu(), wk) and torch.equal(v.cpu(), wv)


def test_a_cache_beyond_32_bits():
    """Offsets past 2^32 bytes and 2^31 elements."""
    k = torch.zeros(1, 5000, 64, 8, 1024, dtype=torch.float16, device="cuda")      # 2.6e9 elements
    v = torch.zeros_like(k)
    k_new, v_new = normal(1, 3, 8, 1024, dtype=torch.float16, seed=8).cuda(), normal(1, 3, 8, 1024, dtype=torch.float16, seed=9).cuda()
    dp.dpllm_cache_append(dp.Cache(k, v, ints([[17, 4999]])), ints([126 - 1]), k_new, v_new)
    assert torch.equal(k[0, 4999, 61:], k_new[0]) and torch.equal(v[0, 4999, 61:], v_new[0])
    assert k.count_nonzero().item() == k_new.count_nonzero().item()


def test_refusals_of_the_binding():
    k = torch.zeros(2, 4, 8, 2, 16, dtype=torch.float16, device="cuda")
    c = dp.Cache(k, k.clone(), ints([[0, 1], [2, 3]]))
    new, lens = torch.zeros(2, 2, 3, 2, 16, dtype=torch.float16, device="cuda"), ints([0, 0])
    for args, kw, word in [((lens, new.float(), new.float()), {}, "type"), ((lens[:1], new, new), {}, "lens"), ((lens, new[..., :8], new[..., :8]), {}, "head_dim"),
                           ((lens, new, new), {"count": ints([1])}, "count"), ((lens, new, new), {"path": ints([[0], [0]])}, "path"),
                           ((lens, new, new), {"layer": 1}, "layers"), ((lens.long(), new, new), {}, "lens")]:
        with pytest.raises(dp.DpllmError, match=word):
            dp.dpllm_cache_append(c, *args, **kw)
    for bad in [(k, k.float()), (k, k[:1]), (k[0], k[0]), (k.transpose(3, 4), k.transpose(3, 4))]:
        with pytest.raises(dp.DpllmError):
            dp.Cache(*bad)
    with pytest.raises(dp.DpllmError, match="table"):
        dp.Cache(k, k, torch.zeros(2, 2, dtype=torch.int64, device="cuda"))
