"""Norms of heads with learned weights and their rotary positions, and the gradient of that, against the formulas in 64 bits on the CPU."""
import pytest
import torch

import paper_2508_06041_amd as dp
from test_gpu_rope import TYPES, normal

pytestmark = pytest.mark.gpu


def turned(y, positions, freqs, scale, layout, back=False):
    """y [batch][tokens][heads][d] in 64 bits, rotated (or by the transpose), and |a| + |b| of the pairs (|y| elsewhere)."""
    if freqs is None:
        return y, y.abs()
    y, r = y.clone(), 2 * freqs.shape[0]
    if positions.dim() == 1:
        positions = positions.expand(y.shape[0], -1)
    t = positions.double().cpu()[:, :, None, None] * freqs.cpu() * (-1.0 if back else 1.0)
    at = (slice(0, r // 2), slice(r // 2, r)) if layout == dp.DPLLM_ROPE_HALF else (slice(0, r, 2), slice(1, r, 2))
    a, b = y[..., at[0]].clone(), y[..., at[1]].clone()
    size = y.abs()
    size[..., at[0]] = size[..., at[1]] = scale * (a.abs() + b.abs())
    y[..., at[0]] = scale * (a * torch.cos(t) - b * torch.sin(t))
    y[..., at[1]] = scale * (a * torch.sin(t) + b * torch.cos(t))
    return y, size


def plain(x, w, positions, freqs, eps, scale=1.0, layout=0):
    """The result and the size its errors go by."""
    y = x.double().cpu()
    y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
    return turned(y if w is None else y * w.double().cpu(), positions, freqs, scale, layout)


def check(got, want, size, dtype):
    """The sum of squares is of at most 32 terms to a lane and 6 levels, so r is good to 2^-19; the rotation to 2^-19 of |a| + |b| (as test_gpu_rope.py
    says); products round in between: 2^-18 in all.  Then the result is rounded to its type."""
    half = torch.finfo(dtype).eps / 2
    err, bound = (got.double().cpu() - want).abs(), size * 2.0 ** -18 + want.abs() * half + 2 * torch.finfo(dtype).smallest_normal * half
    assert (err <= bound).all(), (err - bound).max()


def plain_gradient(x, g, w, positions, freqs, eps, scale=1.0, layout=0):
    """dx and dw of the shape of w (or of heads, d), each with the size its errors go by."""
    x, d = x.double().cpu(), x.shape[-1]
    w = torch.ones(d, dtype=torch.float64) if w is None else w.double().cpu()
    h, size = turned(g.double().cpu(), positions, freqs, scale, layout, back=True)
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    n, e = x * r, h * w
    dx = r * (e - n * (e * n).mean(-1, keepdim=True))
    most = size * w.abs()
    dx_size = r * (most + n.abs() * (most * n.abs()).mean(-1, keepdim=True))
    over = (0, 1) if w.dim() == 2 else (0, 1, 2)
    return dx, dx_size, (h * n).sum(over), (size * n.abs()).sum(over)


def check_gradient(got, x, g, w, *how):
    """dx: the rotation and r as above, twice over, and the mean of d products: 2^-17 of its parts' sizes.  dw: the terms are good to 2^-18, and at most as many rows are added in 32 bits
    one after the other as there are."""
    dx, size, dw, dw_size = plain_gradient(x, g, w, *how)
    half = torch.finfo(x.dtype).eps / 2
    err, bound = (got[0].double().cpu() - dx).abs(), size * 2.0 ** -17 + dx.abs() * half + 2 * torch.finfo(x.dtype).smallest_normal * half
    assert (err <= bound).all(), (err - bound).max()
    if got[1] is not None:
        assert got[1].shape == w.shape and got[1].dtype == w.dtype
        half = torch.finfo(w.dtype).eps / 2
        rows = x.shape[0] * x.shape[1] * (1 if w.dim() == 2 else x.shape[2])
        err, bound = (got[1].double().cpu() - dw).abs(), dw_size * (2.0 ** -18 + (rows + 64) * 2.0 ** -24) + dw.abs() * half + 2 * torch.finfo(w.dtype).smallest_normal * half
        assert (err <= bound).all(), (err - bound).max()


def setup(dtype, batch, tokens, heads, kv, dim, rotary, weights, each, seed=1):
    t = TYPES[dtype]
    xs = tuple((normal(batch, tokens, n, dim, dtype=torch.float32, seed=seed + i) * torch.exp(normal(n, 1, dtype=torch.float32, seed=seed + 9 + i))).to(t) for i, n in enumerate((heads, kv)))
    ws = tuple((1 + 0.5 * normal(*((n,) if each else ()), dim, dtype=torch.float32, seed=seed + 20 + i)).to(TYPES[weights]) for i, n in enumerate((heads, kv)))
    pos = torch.randint(0, 200000, (batch, tokens), generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    freqs, scale = dp.dpllm_rope_frequencies(rotary, 10000.0, dp.DPLLM_ROPE_YARN, 4.0, 4096, 1, 32) if rotary else (None, 1.0)
    return xs, ws, pos, freqs, scale


SHAPES = [(1, 1, 1, 1, 2, 2), (1, 1, 32, 8, 128, 128), (2, 3, 7, 1, 64, 64), (3, 5, 4, 2, 96, 48), (1, 130, 5, 5, 128, 96), (2, 17, 3, 3, 80, 80), (2, 9, 2, 1, 36, 20),
          (1, 4, 1, 1, 1024, 1024), (5, 1, 64, 8, 256, 128), (1, 3, 3, 1, 33, 10), (2, 6, 3, 2, 128, 0), (1, 2, 2, 1, 1, 0), (1, 3, 2, 1, 1023, 0), (3, 700, 2, 1, 64, 64), (1, 3, 2, 2, 1000, 8)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("weights,each", [("f16", False), ("bf16", True), ("f32", False), ("f32", True)])
@pytest.mark.parametrize("shape", SHAPES)
def test_both_ways_against_the_formulas(dtype, layout, weights, each, shape):
    xs, ws, pos, freqs, scale = setup(dtype, *shape, weights, each)
    how = pos, freqs, 1e-3, scale, layout
    outs = dp.dpllm_norm_rope(xs, ws, pos, freqs, eps=1e-3, scale=scale, layout=layout)
    for x, w, o in zip(xs, ws, outs):
        assert o.shape == x.shape and o.dtype == x.dtype
        check(o, *plain(x, w, *how), x.dtype)
    grads = tuple(normal(*x.shape, dtype=x.dtype, seed=40 + i) for i, x in enumerate(xs))
    dx, dw = dp.dpllm_norm_rope_backward(xs, grads, ws, pos, freqs, eps=1e-3, scale=scale, layout=layout)
    for x, g, w, a, b in zip(xs, grads, ws, dx, dw):
        check_gradient((a, b), x, g, w, *how)
    again = dp.dpllm_norm_rope_backward(xs, grads, ws, pos, freqs, eps=1e-3, scale=scale, layout=layout)
    assert all(torch.equal(p, q) for p, q in zip((*dx, *dw), (*again[0], *again[1])))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", [0, 1])
def test_views_in_place_and_shared_positions(dtype, layout):
    """Queries and keys as slices of one projection, heads before tokens, an odd offset, rows with gaps; results in place, gradients over the gradients."""
    t = TYPES[dtype]
    freqs, scale = dp.dpllm_rope_frequencies(64, 5e5)
    pos = torch.arange(1000, 1011, dtype=torch.int32, device="cuda")
    ws = normal(64, dtype=t, seed=8), normal(2, 65, dtype=t, seed=9)[:, 1:]
    for make in (lambda: normal(3, 11, 12, 64, dtype=t, seed=4), lambda: normal(3, 12, 11, 64, dtype=t, seed=5).transpose(1, 2),
                 lambda: normal(3 * 11 * 12 * 64 + 1, dtype=t, seed=6)[1:].view(3, 11, 12, 64), lambda: normal(3, 11, 12, 67, dtype=t, seed=7)[..., :64]):
        x, g = make(), make().mul(0.5)
        before, g_before = x.clone(), g.clone()
        q, k = x[:, :, :8], x[:, :, 8:10]
        gq, gk = g[:, :, :8], g[:, :, 8:10]
        dx, dw = dp.dpllm_norm_rope_backward((q, k), (gq, gk), ws, pos, freqs, layout=layout, out=(gq, gk))
        assert dx[0] is gq
        dp.dpllm_norm_rope((q, k), ws, pos, freqs, out=(q, k), layout=layout)
        for a, z in ((0, 8), (8, 10)):
            w = ws[a // 8]
            check(x[:, :, a:z], *plain(before[:, :, a:z], w, pos, freqs, 1e-6, 1.0, layout), t)
            check_gradient((g[:, :, a:z], dw[a // 8]), before[:, :, a:z], g_before[:, :, a:z], w, pos, freqs, 1e-6, 1.0, layout)
        assert torch.equal(x[:, :, 10:], before[:, :, 10:]) and torch.equal(g[:, :, 10:], g_before[:, :, 10:])


def test_without_weights_and_of_a_lone_tensor():
    x = normal(2, 3, 4, 64, dtype=torch.bfloat16, seed=1)
    check(dp.dpllm_norm_rope(x, None), *plain(x, None, None, None, 1e-6), x.dtype)
    w = normal(64, dtype=torch.float32, seed=2)
    a, b = dp.dpllm_norm_rope((x, x[:, :, :1]), (None, w))
    check(a, *plain(x, None, None, None, 1e-6), x.dtype)
    check(b, *plain(x[:, :, :1], w, None, None, 1e-6), x.dtype)
    g = normal(2, 3, 4, 64, dtype=torch.bfloat16, seed=3)
    dx, dw = dp.dpllm_norm_rope_backward((x, x), (g, g), (None, w))
    assert dw[0] is None
    check_gradient((dx[0], None), x, g, None, None, None, 1e-6)
    check_gradient((dx[1], dw[1]), x, g, w, None, None, 1e-6)
    assert dp.dpllm_norm_rope_backward(x, g, w, wanted=[False])[1] is None
    dx, dw = dp.dpllm_norm_rope_backward(x[:0], g[:0], w)      # no tokens: no gradient
    assert dx.shape[0] == 0 and (dw == 0).all()
    big = torch.full((1, 1, 1, 64), 3e38, device="cuda")       # the sum of squares is infinite, as in the formula in 32 bits
    assert (dp.dpllm_norm_rope(big, None) == 0).all()
    zero = torch.zeros(1, 1, 1, 64, device="cuda")
    assert (dp.dpllm_norm_rope(zero, None) == 0).all() and torch.isnan(dp.dpllm_norm_rope(zero, None, eps=0.0)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_through_autograd(dtype):
    (q, k), (wq, wk), pos, freqs, scale = setup(dtype, 2, 5, 6, 2, 64, 48, "f32", False)
    want = dp.dpllm_norm_rope((q, k), (wq, wk), pos, freqs, scale=scale)
    assert not want[0].requires_grad
    for t in (q, k, wq, wk):
        t.requires_grad_()
    outs = dp.dpllm_norm_rope((q, k), (wq, wk), pos, freqs, scale=scale)
    assert all(torch.equal(a, b) and a.requires_grad for a, b in zip(outs, want))
    grads = [normal(*o.shape, dtype=o.dtype, seed=4 + i) for i, o in enumerate(outs)]
    torch.autograd.backward(outs, grads)
    for x, w, g in ((q, wq, grads[0]), (k, wk, grads[1])):
        check_gradient((x.grad, w.grad), x.detach(), g, w.detach(), pos, freqs, 1e-6, scale)
    # some of them, and a gradient that is one number for all
    q, k, wq, wk = (t.detach() for t in (q, k, wq, wk))
    wk = wk.clone().requires_grad_()
    a, b = dp.dpllm_norm_rope((q, k), (wq, wk), pos, freqs, scale=scale)
    (a.float().sum() + b.float().sum()).backward()
    assert q.grad is None or not q.requires_grad
    check_gradient((plain_gradient(k, torch.ones_like(k), wk.detach(), pos, freqs, 1e-6, scale)[0], wk.grad), k, torch.ones_like(k), wk.detach(), pos, freqs, 1e-6, scale)
    y = dp.dpllm_norm_rope(q.clone().requires_grad_(), None, pos, freqs, scale=scale)      # a lone tensor, no weight
    assert y.requires_grad and isinstance(y, torch.Tensor)
    y.float().sum().backward()
    with pytest.raises(dp.DpllmError, match="out"):
        dp.dpllm_norm_rope(q.clone().requires_grad_(), None, pos, freqs, out=q.clone())


@pytest.mark.parametrize("layout", [0, 1])
def test_against_differences(layout):
    """Central differences are off by c h^2, which two steps tell, and by the rounding of the values over the step."""
    (x, _), (w, _), pos, freqs, scale = setup("f32", 2, 3, 4, 1, 64, 48, "f32", True)
    g, dx, dw = (normal(*t.shape, dtype=torch.float32, seed=s) for t, s in ((x, 5), (x, 6), (w, 7)))

    def value(y, v):
        return (dp.dpllm_norm_rope(y, v, pos, freqs, scale=scale, layout=layout).double() * g.double()).sum().item()
    grad_x, grad_w = dp.dpllm_norm_rope_backward(x, g, w, pos, freqs, scale=scale, layout=layout)
    size = (plain(x, w, pos, freqs, 1e-6, scale, layout)[1] * g.double().cpu().abs()).sum().item()
    for slope, move in (((grad_x.double() * dx.double()).sum().item(), lambda h: (x + h * dx, w)), ((grad_w.double() * dw.double()).sum().item(), lambda h: (x, w + h * dw))):
        def difference(h):
            return (value(*move(h)) - value(*move(-h))) / (2 * h)
        wide, narrow = difference(2.0 ** -6), difference(2.0 ** -7)
        assert abs(narrow - slope) <= abs(wide - narrow) + 2 * size * 2.0 ** -18 * 2.0 ** 7


def test_many_tokens_and_graphs():
    """More tokens than a grid of workgroups takes at once, and both directions captured and replayed."""
    xs, ws, pos, freqs, scale = setup("bf16", 2, 3000, 3, 1, 128, 128, "f32", False)
    grads = tuple(normal(*x.shape, dtype=x.dtype, seed=40 + i) for i, x in enumerate(xs))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def step():
        return dp.dpllm_norm_rope(xs, ws, pos, freqs, scale=scale), dp.dpllm_norm_rope_backward(xs, grads, ws, pos, freqs, scale=scale)
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs, (dx, dw) = step()
    for i in range(4):
        for x, g, w in zip(xs, grads, ws):
            x.copy_(normal(*x.shape, dtype=x.dtype, seed=50 + i))
            g.mul_(-0.5)
            w.add_(0.125)
        pos.add_(17)
        want, (want_dx, want_dw) = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*outs, *dx, *dw), (*want, *want_dx, *want_dw)))
    check_gradient((dx[0], dw[0]), xs[0], grads[0], ws[0], pos, freqs, 1e-6, scale)
