"""Attention of drafted tokens over a paged cache against the formula in 64 bits."""
import math

import pytest
import torch

import paper_2508_06041_amd as dp

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def normal(*shape, dtype, seed, size=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * size).to(dtype)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def words(sees):
    """int64 [batch][nodes][ceil(nodes / 64)] of a bool [batch][nodes][nodes]."""
    b, n, _ = sees.shape
    m = torch.zeros(b, n, (n + 63) // 64, dtype=torch.int64)
    for j in range(n):
        m[:, :, j // 64] |= sees[:, :, j].long() << (j % 64)
    return m.cuda()


class Case:
    """Inputs on the CPU, and the answer in 64 bits with how far off it may be."""

    def __init__(self, dtype, batch, nodes, heads, kv, dim, page, lens, mask="chain", seed=1, size=1.0, spare=3, new=True, scale=None):
        g = torch.Generator().manual_seed(seed)
        self.t = TYPES[dtype]
        self.scale = dim ** -0.5 if scale is None else scale
        each = max(1, -(-max(lens) // page))
        pages = batch * each + spare
        self.k, self.v = (normal(1, pages, page, kv, dim, dtype=self.t, seed=seed + i) for i in (1, 2))
        self.table = torch.randperm(pages, generator=g)[:batch * each].reshape(batch, each).to(torch.int32)
        self.lens = lens
        self.q = normal(batch, nodes, heads, dim, dtype=self.t, seed=seed + 3, size=size)
        self.k_new, self.v_new = (normal(batch, nodes, kv, dim, dtype=self.t, seed=seed + i) if new else None for i in (4, 5))
        if mask == "chain":
            self.sees = torch.ones(nodes, nodes, dtype=torch.bool).tril()[None].expand(batch, -1, -1)
        elif mask == "tree":
            self.sees = torch.zeros(batch, nodes, nodes, dtype=torch.bool)
            for b in range(batch):
                for i in range(nodes):
                    if i:
                        self.sees[b, i] = self.sees[b, int(torch.randint(0, i, (1,), generator=g))]
                    self.sees[b, i, i] = True
        else:                                    # anything, rows that see no node among it
            self.sees = torch.rand(batch, nodes, nodes, generator=g) < 0.3
            self.sees[:, ::3] = False
        self.mask = None if mask == "chain" else words(self.sees)

    def plain(self):
        b, n, h, d = self.q.shape
        kv = self.k.shape[3]
        out, lse = torch.zeros(b, n, h, d, dtype=torch.float64), torch.zeros(b, n, h, dtype=torch.float64)
        self.bound, self.lse_bound = torch.zeros_like(out), torch.zeros_like(lse)
        eps = torch.finfo(self.t).eps / 2
        pool_k, pool_v = self.k[0].double().cuda(), self.v[0].double().cuda()
        for s in range(b):
            ids = self.table[s].tolist()
            ok = torch.tensor([0 <= i < self.k.shape[1] for i in ids]).repeat_interleave(self.k.shape[2])
            ids = [i if 0 <= i < self.k.shape[1] else 0 for i in ids]
            length = max(0, min(self.lens[s], ok.numel()))
            ok = ok[:length]
            keys, values = (p[ids].flatten(0, 1)[:length] for p in (pool_k, pool_v))
            sees = ok[None].expand(n, length)
            if self.k_new is not None:
                keys, values = torch.cat([keys, self.k_new[s].double().cuda()]), torch.cat([values, self.v_new[s].double().cuda()])
                sees = torch.cat([sees, self.sees[s]], dim=1)
            sees = sees.cuda()
            for i in range(h):
                q, k, v = self.q[s, :, i].double().cuda(), keys[:, i * kv // h], values[:, i * kv // h]
                x = (q @ k.t().contiguous() * self.scale).masked_fill(~sees, -math.inf)
                size = (q.abs() @ k.abs().t().contiguous() * abs(self.scale)).masked_fill(~sees, 0.0)
                for r in range(n):               # only what the row sees, so that anything may stand elsewhere
                    at = sees[r]
                    if not at.any():
                        lse[s, r, i] = -math.inf
                        continue
                    y, w = x[r, at], v[at]
                    p = torch.softmax(y, 0)
                    o = p @ w
                    out[s, r, i], lse[s, r, i] = o.cpu(), torch.logsumexp(y, 0).cpu()
                    # a score is a sum of d products in 32 bits, and an exponent's error is a weight's relative one, in numerator and denominator; the
                    # weight is rounded to the type (half a step), the sums over the tokens are in 32 bits, then the result is rounded
                    score = 2.0 ** -23 * (d + 4) * size[r, at].max().item() + 2.0 ** -20
                    some = eps + 2 * score + 2 * at.sum().item() * 2.0 ** -24
                    self.bound[s, r, i] = (some * (p @ w.abs()) + eps * o.abs()).cpu() + torch.finfo(self.t).smallest_normal * eps
                    self.lse_bound[s, r, i] = score + at.sum().item() * 2.0 ** -24 + 2.0 ** -22 * (1 + abs(lse[s, r, i].item()))
        return out, lse

    def run(self, **kw):
        def dev(x):
            return None if x is None else x.cuda()
        k, v = self.k.cuda(), self.v.cuda()
        lse = torch.full(self.q.shape[:3], math.nan, device="cuda")
        kw = {"max_len": max(self.lens), **kw}
        out = dp.dpllm_tree_attention(dp.Cache(k, v, self.table.cuda()), 0, ints(self.lens), dev(self.q), dev(self.k_new), dev(self.v_new), mask=self.mask,
                                      scale=self.scale, lse=lse, **kw)
        return out, lse

    def check(self, **kw):
        out, lse = self.run(**kw)
        want, want_lse = self.plain()
        err = (out.double().cpu() - want).abs()
        assert (err <= self.bound).all(), ((err / self.bound).max(), err.max())
        none = want_lse == -math.inf
        assert torch.equal(lse.cpu() == -math.inf, none)
        assert ((lse.double().cpu() - want_lse).abs()[~none] <= self.lse_bound[~none]).all()
        assert (out.cpu()[none] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("nodes,heads,kv", [(1, 1, 1), (1, 8, 2), (5, 6, 1), (13, 4, 4), (33, 6, 2)])
@pytest.mark.parametrize("page,lens", [(16, [0, 1]), (32, [31, 129]), (1, [5, 40]), (7, [100, 33]), (64, [700, 64])])
def test_types_heads_and_pages(dtype, dim, nodes, heads, kv, page, lens):
    Case(dtype, 2, nodes, heads, kv, dim, page, lens, mask="tree").check()


@pytest.mark.parametrize("mask", ["chain", "tree", "any"])
@pytest.mark.parametrize("nodes", [2, 8, 31, 32, 64, 65, 129, 256])
def test_masks(mask, nodes):
    Case("bf16", 2, nodes, 4, 2, 128, 16, [0, 45], mask=mask, seed=nodes).check()


def test_a_mask_for_all_sequences():
    c = Case("f16", 3, 9, 4, 2, 64, 16, [3, 0, 70], mask="tree")
    c.sees = c.sees[:1].expand(3, -1, -1)
    c.mask = c.mask[:1].contiguous()
    c.check()


@pytest.mark.parametrize("lens", [[0, 0], [0, 3], [-5, 100]])
@pytest.mark.parametrize("nodes", [1, 4])
def test_the_cache_only(lens, nodes):
    """No new keys; sequences without a token give zeros."""
    Case("f16", 2, nodes, 8, 2, 128, 16, lens, new=False).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("max_len", [0, 1, 3000, 100000])
def test_long_and_ragged_contexts_however_split(dtype, max_len):
    Case(dtype, 5, 3, 8, 2, 128, 64, [2999, 1, 0, 1024, 1531], mask="tree").check(max_len=max_len)


@pytest.mark.parametrize("page", [1, 8, 16, 32, 33, 64])
def test_bad_pages_hold_nothing(page):
    c = Case("bf16", 3, 4, 4, 2, 128, page, [200, 130, 77], mask="tree")
    c.table[0, 0] = -1
    c.table[1, -1] = c.k.shape[1]
    c.table[2, c.table.shape[1] // 4] = 2 ** 31 - 1
    c.check()
    c.table[1] = -7                       # not one page
    c.check()


def test_lengths_past_the_pages_are_cut():
    c = Case("f16", 2, 2, 4, 2, 64, 16, [40, 20])
    c.lens = [1000, 2 ** 31 - 1]
    c.check(max_len=48)


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_seen_may_be_anything(dtype):
    """NaN and infinities in pages of nobody, behind the lengths, and in nodes that a row does not see."""
    c = Case(dtype, 3, 40, 4, 2, 128, 16, [45, 0, 16], mask="any", seed=3)
    used = torch.zeros(c.k.shape[1:3], dtype=torch.bool)
    for s, length in enumerate(c.lens):
        for t in range(length):
            used[c.table[s, t // 16], t % 16] = True
    c.k[0, ~used] = math.nan
    c.v[0, ~used] = math.inf
    c.sees[:, :, 7] = c.sees[:, :, 39] = False
    c.mask = words(c.sees)
    for j, value in ((7, math.nan), (39, math.inf)):
        c.k_new[:, j] = value
        c.v_new[:, j, :, ::3] = value
    c.check()
    # a node that some rows see: they get what it holds, the others nothing of it
    c.sees[:, 1::6, 7] = True
    c.mask = words(c.sees)
    c.k_new[:, 7] = 0.5
    c.v_new[:, 7] = -1.0
    c.v_new[:, 7, :, 5], c.v_new[:, 7, :, 64] = -math.inf, math.nan
    out = c.run()[0].cpu()
    hit = c.sees[:, :, 7]
    assert (out[hit][..., 5] == -math.inf).all() and out[hit][..., 64].isnan().all()
    assert out[~hit].isfinite().all() and out[hit][..., [0, 4, 6, 63, 65, 127]].isfinite().all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("nodes,length", [(6, 40), (6, 3000), (14, 40), (14, 3000), (70, 3000)])
def test_odd_values_of_nodes_however_many_rows(dtype, dim, nodes, length):
    """The same in every kernel, in one part and in several: an infinity and a NaN that some rows see, and what nobody does."""
    c = Case(dtype, 2, nodes, 4, 2, dim, 16, [length, 5], mask="any", seed=nodes)
    some, none = 2, nodes - 1
    c.sees[:, :, some] = c.sees[:, :, none] = False
    c.mask = words(c.sees)
    c.k_new[:, none], c.v_new[:, none] = math.nan, -math.inf
    c.check()
    c.sees[:, 1::2, some] = True
    c.mask = words(c.sees)
    c.v_new[:, some, :, 7], c.v_new[:, some, :, dim - 1] = math.inf, math.nan
    out = c.run()[0].cpu()
    hit = c.sees[:, :, some]
    assert (out[hit][..., 7] == math.inf).all() and out[hit][..., dim - 1].isnan().all()
    assert out[~hit].isfinite().all()
    c.v_new[:, some, :, 7] = c.v_new[:, some, :, dim - 1] = 0.0
    want, _ = c.plain()
    rest = [i for i in range(dim) if i not in (7, dim - 1)]
    assert ((out.double() - want).abs()[..., rest] <= c.bound[..., rest]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_far_apart(dtype):
    """Scores of hundreds; a row whose every score is far below zero; one token that carries all and many that carry little each."""
    Case(dtype, 1, 4, 4, 2, 128, 16, [300], size=30.0).check()
    c = Case(dtype, 1, 2, 2, 1, 64, 16, [500], new=False)
    c.q[:] = 1.0
    c.k[:] = -40.0
    c.check()
    c = Case(dtype, 1, 1, 1, 1, 64, 64, [20000], new=False)
    c.q[:] = 0.0
    c.k[:] = 0.0
    c.v[:] = 1.0
    c.q[..., 0], c.scale = 1.0, 1.0
    c.k[..., 0] = -17.5                    # 20000 e^-17.5 = 5e-4 of the one token's weight: values of 1 against its 0
    at = c.table[0, 0].item()
    c.k[0, at, 0, 0, 0], c.v[0, at, 0] = 0.0, 0.0
    c.check()


def test_the_lowest_value_is_a_number():
    """A score of the type's lowest value counts as any other."""
    c = Case("bf16", 1, 1, 1, 1, 64, 16, [16], new=False, scale=1.0)
    c.q[:], c.k[:] = 0.0, 0.0
    c.q[..., 0] = 1.0
    c.k[..., 0] = torch.finfo(torch.bfloat16).min
    out, lse = c.run()
    assert torch.allclose(out.double().cpu(), c.v[0, c.table[0, 0]].double().mean(0)[None, None], atol=2 ** -8)
    assert lse.item() == pytest.approx(torch.finfo(torch.bfloat16).min, rel=2 ** -8)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30, 3.0])
@pytest.mark.parametrize("nodes", [3, 40])
def test_scales(dtype, scale, nodes):
    """Negative ones turn the order round, 0 makes all weights equal."""
    Case(dtype, 2, nodes, 4, 2, 128, 16, [333, 0], mask="tree", scale=scale).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_views(dtype):
    """Queries, keys and values as slices of one projection, heads before tokens in the results, pages that hold head after head."""
    c = Case(dtype, 2, 5, 6, 2, 128, 16, [37, 90], mask="tree")
    want, _ = c.run()
    qkv = torch.cat([c.q, c.k_new, c.v_new], dim=2).cuda()
    out = torch.empty(2, 6, 5, 128, dtype=c.t, device="cuda").transpose(1, 2)
    k, v = (x.transpose(2, 3).contiguous().cuda().transpose(2, 3) for x in (c.k, c.v))
    wide = torch.full((2, c.table.shape[1] + 3), -1, dtype=torch.int32, device="cuda")
    wide[:, :-3] = c.table
    got = dp.dpllm_tree_attention(dp.Cache(k, v, wide[:, :-3]), 0, ints(c.lens), qkv[:, :, :6], qkv[:, :, 6:8], qkv[:, :, 8:], mask=c.mask, out=out, max_len=90)
    assert got is out and torch.equal(out, want)


def test_layers_and_no_table():
    """The second layer of a cache with one stretch per sequence, of a length that is no multiple of anything."""
    c = Case("f16", 2, 3, 4, 2, 64, 77, [77, 50], spare=0)
    c.table = torch.tensor([[0], [1]], dtype=torch.int32)
    want, _ = c.run()
    k, v = (torch.cat([torch.full_like(x, math.nan), x]).cuda() for x in (c.k, c.v))
    got = dp.dpllm_tree_attention(dp.Cache(k, v), 1, ints(c.lens), c.q.cuda(), c.k_new.cuda(), c.v_new.cuda(), max_len=77)
    assert torch.equal(got, want)


def test_a_cache_beyond_32_bits():
    k = torch.zeros(1, 4200, 64, 32, 256, dtype=torch.float16, device="cuda")       # 2.2e9 elements
    v = torch.zeros_like(k)
    k[0, 4199], v[0, 4199] = normal(64, 32, 256, dtype=torch.float16, seed=1).cuda(), normal(64, 32, 256, dtype=torch.float16, seed=2).cuda()
    q = normal(1, 2, 32, 256, dtype=torch.float16, seed=3).cuda()
    got = dp.dpllm_tree_attention(dp.Cache(k, v, ints([[4199]])), 0, ints([60]), q)
    small = dp.dpllm_tree_attention(dp.Cache(k[:, 4199:].clone(), v[:, 4199:].clone(), ints([[0]])), 0, ints([60]), q)
    assert torch.equal(got, small) and got.count_nonzero() > 0


def test_the_same_bits_twice_and_in_a_graph():
    c = Case("bf16", 4, 7, 16, 4, 128, 16, [4000, 17, 1000, 0], mask="tree")
    out, lse = c.run()
    again, _ = c.run()
    assert torch.equal(out, again)
    cache, lens = dp.Cache(c.k.cuda(), c.v.cuda(), c.table.cuda()), ints(c.lens)
    q, k, v, into = c.q.cuda(), c.k_new.cuda(), c.v_new.cuda(), torch.empty_like(out)
    need = dp.dpllm_tree_attention_workspace_bytes(4, 7, 16, 4, 128, 4000)
    assert need > 0
    space = torch.empty(need, dtype=torch.uint8, device="cuda")

    def go():
        dp.dpllm_tree_attention(cache, 0, lens, q, k, v, mask=c.mask, out=into, max_len=4000, workspace=space)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    side.synchronize()
    assert torch.equal(into, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for new in ([4000, 17, 1000, 0], [1, 0, 64, 4000], [333, 4000, 0, 31]):
        c.lens = new
        lens.copy_(torch.tensor(new))
        space.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(into, c.run(max_len=4000)[0])


def test_refusals_of_the_binding():
    c = Case("f16", 2, 3, 4, 2, 64, 16, [40, 20])
    cache, lens, q, k, v = dp.Cache(c.k.cuda(), c.v.cuda(), c.table.cuda()), ints(c.lens), c.q.cuda(), c.k_new.cuda(), c.v_new.cuda()
    for args, kw, word in [((lens, q.float(), k, v), {}, "type"), ((lens[:1], q, k, v), {}, "lens"), ((lens, q, k, None), {}, "together"),
                           ((lens, q, k[:, :2], v[:, :2]), {}, "k_new"), ((lens, q, k, v), {"mask": torch.zeros(2, 3, 1, device="cuda")}, "mask"),
                           ((lens, q, k, v), {"mask": torch.zeros(2, 3, 2, dtype=torch.int64, device="cuda")}, "mask"),
                           ((lens, q, k, v), {"lse": torch.zeros(2, 3, device="cuda")}, "lse"), ((lens, q, k, v), {"out": q[:, :2]}, "out"),
                           ((lens, q[:, :, :3], k, v), {}, "heads"), ((lens, q, k, v), {"scale": math.nan}, "scale")]:
        with pytest.raises(dp.DpllmError, match=word):
            dp.dpllm_tree_attention(cache, 0, *args, **kw)
    far = dp.Cache(cache.k, cache.v, cache.table.repeat(1, 100))      # 4800 tokens: the work is split
    with pytest.raises(dp.DpllmError, match="workspace"):
        dp.dpllm_tree_attention(far, 0, lens, q, k, v, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(dp.DpllmError, match="layer"):
        dp.dpllm_tree_attention(cache, 1, lens, q, k, v)
    assert dp.dpllm_tree_attention(cache, 0, lens[:0], q[:0], k[:0], v[:0]).shape == (0, 3, 4, 64)
    assert dp.dpllm_tree_attention(cache, 0, lens, q[:, :0], k[:, :0], v[:, :0]).shape == (2, 0, 4, 64)
