"""The gradient of rotary positions through autograd, against the formula's and against differences."""
import pytest
import torch

import paper_2508_06041_amd as dp
from test_gpu_rope import TYPES, check, normal, plain

pytestmark = pytest.mark.gpu


def setup(dtype, batch=2, tokens=5, heads=6, kv=2, dim=64, rotary=48):
    t = TYPES[dtype]
    q, k = normal(batch, tokens, heads, dim, dtype=t, seed=1), normal(batch, tokens, kv, dim, dtype=t, seed=2)
    pos = torch.randint(0, 20000, (batch, tokens), generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    return q, k, pos, *dp.dpllm_rope_frequencies(rotary, 10000.0, dp.DPLLM_ROPE_YARN, 4.0, 4096, 1, 32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("inverse", [False, True])
def test_against_the_formula(dtype, layout, inverse):
    q, k, pos, freqs, scale = setup(dtype)
    want = dp.dpllm_rope((q, k), pos, freqs, scale=scale, layout=layout, inverse=inverse)
    assert not want[0].requires_grad
    q.requires_grad_()
    k.requires_grad_()
    outs = dp.dpllm_rope((q, k), pos, freqs, scale=scale, layout=layout, inverse=inverse)
    assert all(torch.equal(a, b) and a.requires_grad for a, b in zip(outs, want))
    grads = [normal(*o.shape, dtype=o.dtype, seed=4 + i) for i, o in enumerate(outs)]
    torch.autograd.backward(outs, grads)
    for x, g in ((q, grads[0]), (k, grads[1])):
        assert x.grad.dtype == x.dtype
        check(x.grad, *plain(g, pos, freqs, scale, layout, not inverse), x.dtype)


@pytest.mark.parametrize("layout", [0, 1])
def test_against_differences(layout):
    """The map is linear: the difference over any step is the gradient, to the rounding of the results."""
    q, _, pos, freqs, scale = setup("f32")
    g, d = normal(*q.shape, dtype=torch.float32, seed=7), normal(*q.shape, dtype=torch.float32, seed=8)

    def value(x):
        return (dp.dpllm_rope(x, pos, freqs, scale=scale, layout=layout).double() * g.double()).sum()
    moved = (value(q + d) - value(q - d)).item() / 2
    q.requires_grad_()
    value(q).backward()
    size = (g.double().abs() * (d.double().abs() + q.detach().double().abs())).sum().item()
    assert abs(moved - (q.grad.double() * d.double()).sum().item()) <= 2.0 ** -17 * size      # every term is good to 2^-19 of its pair's size


def test_some_of_the_tensors_and_lone_ones():
    q, k, pos, freqs, scale = setup("f32")
    k.requires_grad_()
    a, b = dp.dpllm_rope((q, k), pos, freqs, scale=scale)
    (a.sum() + (2 * b).sum()).backward()                       # gradients without strides
    assert q.grad is None
    check(k.grad, *plain(torch.full_like(k, 2.0), pos, freqs, scale, 0, True), torch.float32)
    q.requires_grad_()
    one = dp.dpllm_rope(q, pos[0], freqs, scale=scale)         # shared positions
    assert isinstance(one, torch.Tensor)
    g, = torch.autograd.grad(one, q, one.detach())
    check(g, *plain(one.detach(), pos[:1].expand(2, -1), freqs, scale, 0, True), torch.float32)
    with torch.no_grad():
        assert not dp.dpllm_rope(q, pos, freqs, scale=scale).requires_grad


def test_the_gradient_of_the_gradient():
    q, _, pos, freqs, scale = setup("f32")
    g = normal(*q.shape, dtype=torch.float32, seed=9).requires_grad_()
    q.requires_grad_()
    back, = torch.autograd.grad(dp.dpllm_rope(q, pos, freqs, scale=scale), q, g, create_graph=True)
    h = normal(*q.shape, dtype=torch.float32, seed=10)
    again, = torch.autograd.grad(back, g, h)
    check(again, *plain(h, pos, freqs, scale, 0, False), torch.float32)


def test_positions_that_changed_behind_the_call_are_noticed():
    q, _, pos, freqs, scale = setup("f32")
    out = dp.dpllm_rope(q.requires_grad_(), pos, freqs, scale=scale)
    pos += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_a_gradient_and_a_place_for_the_results():
    q, k, pos, freqs, scale = setup("f16")
    into = torch.empty_like(q)
    for x, out in ((q.clone().requires_grad_(), into), (q, into.clone().requires_grad_())):
        with pytest.raises(dp.DpllmError, match="gradient"):
            dp.dpllm_rope(x, pos, freqs, out=out, scale=scale)
        with torch.no_grad():
            assert dp.dpllm_rope(x, pos, freqs, out=out, scale=scale) is out
