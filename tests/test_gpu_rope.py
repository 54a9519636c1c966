"""Rotary positions against the formula in 64 bits on the CPU."""
import math

import pytest
import torch

import paper_2508_06041_amd as dp

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def plain(x, positions, freqs, scale, layout, inverse):
    """x: [batch][tokens][heads][d] of any type; positions [batch][tokens]."""
    y, r = x.double().cpu(), 2 * freqs.shape[0]
    t = positions.double().cpu()[:, :, None, None] * freqs.cpu() * (-1.0 if inverse else 1.0)
    at = (slice(0, r // 2), slice(r // 2, r)) if layout == dp.DPLLM_ROPE_HALF else (slice(0, r, 2), slice(1, r, 2))
    a, b = y[..., at[0]].clone(), y[..., at[1]].clone()
    y[..., at[0]] = scale * (a * torch.cos(t) - b * torch.sin(t))
    y[..., at[1]] = scale * (a * torch.sin(t) + b * torch.cos(t))
    size = torch.zeros_like(y)      # |a| + |b| of the pair
    size[..., at[0]] = size[..., at[1]] = scale * (a.abs() + b.abs())
    return y, size


def check(got, want, size, dtype):
    """The angle in turns is rounded to a float (2^-26 turns, 9.4e-8 in the sine), sine and cosine are good to a few 2^-24, two products and a sum
    round, and an angle of 2^31 radians is off by 4.8e-7: 2^-19 of |a| + |b| in all; then the result is rounded to its type."""
    bound = size * 2.0 ** -19 + want.abs() * (torch.finfo(dtype).eps / 2) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    err = (got.double().cpu() - want).abs()
    assert (err <= bound).all(), (err - bound).max()


def normal(*shape, dtype, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("batch,tokens,heads,kv,dim,rotary", [
    (1, 1, 1, 1, 2, 2), (1, 1, 32, 8, 128, 128), (2, 3, 7, 1, 64, 64), (3, 5, 4, 2, 96, 48), (1, 130, 5, 5, 128, 96), (2, 17, 3, 3, 80, 80), (2, 9, 2, 1, 36, 20),
    (1, 4, 1, 1, 1024, 1024), (5, 1, 64, 8, 256, 128), (1, 3, 3, 1, 33, 10)])
def test_against_the_formula(dtype, layout, inverse, batch, tokens, heads, kv, dim, rotary):
    t = TYPES[dtype]
    q, k = normal(batch, tokens, heads, dim, dtype=t, seed=1), normal(batch, tokens, kv, dim, dtype=t, seed=2)
    pos = torch.randint(0, 200000, (batch, tokens), generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    freqs, scale = dp.dpllm_rope_frequencies(rotary, 10000.0, dp.DPLLM_ROPE_YARN, 4.0, 4096, 1, 32)
    out = dp.dpllm_rope((q, k), pos, freqs, scale=scale, layout=layout, inverse=inverse)
    for x, o in zip((q, k), out):
        assert o.shape == x.shape and o.dtype == t
        check(o, *plain(x, pos, freqs, scale, layout, inverse), t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", [0, 1])
def test_views_in_place_and_shared_positions(dtype, layout):
    """Queries and keys as slices of one projection, heads before tokens, an odd offset, results in place."""
    t = TYPES[dtype]
    freqs, scale = dp.dpllm_rope_frequencies(64, 5e5, dp.DPLLM_ROPE_BANDS, 8.0, 8192, 1, 4)
    pos = torch.arange(1000, 1011, dtype=torch.int32, device="cuda")
    for make in (lambda: normal(3, 11, 12, 64, dtype=t, seed=4),                              # sliced along the heads
                 lambda: normal(3, 12, 11, 64, dtype=t, seed=5).transpose(1, 2),              # head after head
                 lambda: normal(3 * 11 * 12 * 64 + 1, dtype=t, seed=6)[1:].view(3, 11, 12, 64),   # no 16-byte alignment
                 lambda: normal(3, 11, 12, 67, dtype=t, seed=7)[..., :64]):                   # rows that are no multiple of 16 bytes
        x = make()
        before = x.clone()
        q, k = x[:, :, :8], x[:, :, 8:10]
        dp.dpllm_rope((q, k), pos, freqs, out=(q, k), scale=scale, layout=layout)
        want, size = plain(before, pos.expand(3, 11), freqs, scale, layout, False)
        check(x[:, :, :10], want[:, :, :10], size[:, :, :10], t)
        assert torch.equal(x[:, :, 10:], before[:, :, 10:])


def test_far_and_negative_positions():
    x = normal(1, 6, 2, 128, dtype=torch.float32, seed=8)
    pos = torch.tensor([[0, -1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 131071]], dtype=torch.int32, device="cuda")
    freqs, scale = dp.dpllm_rope_frequencies(128)
    assert scale == 1.0
    check(dp.dpllm_rope(x, pos, freqs), *plain(x, pos, freqs, 1.0, 0, False), torch.float32)


@pytest.mark.parametrize("layout", [0, 1])
def test_the_inverse_is_the_gradient(layout):
    """<g, rope(x + d) - rope(x - d)> / 2 = <inverse(g), d>, and it undoes a rotation without scale."""
    n = (2, 5, 3, 64)
    x, g, d = normal(*n, dtype=torch.float32, seed=9), normal(*n, dtype=torch.float32, seed=10), normal(*n, dtype=torch.float32, seed=11)
    pos = torch.arange(10, dtype=torch.int32, device="cuda").reshape(2, 5) * 77
    freqs, scale = dp.dpllm_rope_frequencies(48, 10000.0, dp.DPLLM_ROPE_YARN, 16.0, 2048, 1, 32)

    def f(y):
        return dp.dpllm_rope(y, pos, freqs, scale=scale, layout=layout).double()
    moved = (g.double() * (f(x + d) - f(x - d))).sum().item() / 2
    back = dp.dpllm_rope(g, pos, freqs, scale=scale, layout=layout, inverse=True).double()
    # every one of the 1920 terms is good to 2^-19 of its size, about 1.7 in the mean
    assert abs(moved - (back * d.double()).sum().item()) <= 2.0 ** -18 * 2 * (g.double().abs() * (d.double().abs() + x.double().abs())).sum().item()
    same = dp.dpllm_rope(dp.dpllm_rope(x, pos, freqs, layout=layout), pos, freqs, layout=layout, inverse=True)
    check(same, x.double().cpu(), 4 * x.double().abs().amax(-1, keepdim=True).expand(n).cpu(), torch.float32)


def test_nothing_and_many_tokens():
    freqs, _ = dp.dpllm_rope_frequencies(8)
    assert dp.dpllm_rope(torch.empty(0, 4, 2, 8, device="cuda"), torch.empty(0, 4, dtype=torch.int32, device="cuda"), freqs).shape == (0, 4, 2, 8)
    assert dp.dpllm_rope(torch.empty(3, 0, 2, 8, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), freqs).shape == (3, 0, 2, 8)
    n = 5_000_003      # more tokens than a grid has workgroups for
    x = normal(1, n, 1, 8, dtype=torch.float16, seed=12)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    got = dp.dpllm_rope(x, pos, freqs)
    for part in (slice(0, 1000), slice(n // 2, n // 2 + 1000), slice(n - 1000, n)):
        check(got[:, part], *plain(x[:, part], pos[None, part], freqs, 1.0, 0, False), torch.float16)


def test_a_graph_follows_the_positions():
    x = normal(2, 4, 6, 128, dtype=torch.bfloat16, seed=13)
    pos = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    freqs, _ = dp.dpllm_rope_frequencies(128)
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        dp.dpllm_rope(x, pos, freqs, out=out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dp.dpllm_rope(x, pos, freqs, out=out)
    for i in range(4):
        pos.copy_(torch.randint(0, 9999, (2, 4), generator=torch.Generator().manual_seed(i)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, dp.dpllm_rope(x, pos, freqs))


def test_refusals_of_the_binding():
    freqs, _ = dp.dpllm_rope_frequencies(8)
    x, pos = torch.zeros(1, 2, 3, 8, device="cuda"), torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    for args, word in [((x.double(), pos, freqs), "float16"), ((x.cpu(), pos, freqs), "device"), ((x, pos.long(), freqs), "positions"),
                       ((x, pos[:, :1], freqs), "positions"), ((x, pos, freqs.float()), "freqs"), (((x, x.half()), pos, freqs), "share"),
                       ((x.transpose(2, 3), pos, freqs), "contiguous"), ((x[0], pos, freqs), "batch"), (((x,) * 5, pos, freqs), "1 to 4"),
                       ((x[..., :4].contiguous(), pos, freqs), "rotary_dim")]:
        with pytest.raises(dp.DpllmError, match=word):
            dp.dpllm_rope(*args)
    with pytest.raises(dp.DpllmError, match="out"):
        dp.dpllm_rope(x, pos, freqs, out=(x, x))
    assert math.isfinite(dp.dpllm_rope(x, pos, freqs).sum().item())
