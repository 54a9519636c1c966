"""Attention over a quantised cache: how far weights are rounded, of the cached tokens and of the new ones, told from results in which values cancel."""
import math

import pytest
import torch

from test_gpu_quantized_attention import Case
from test_gpu_quantized_cache import FORMS, decoded
from test_gpu_tree_attention import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length,nodes,new", [(700, 1, False), (0, 200, True), (90, 60, True), (300, 13, False), (0, 40, True), (33, 30, True)])
@pytest.mark.parametrize("dim", [64, 128])
def test_weights_keep_16_bits(form, dtype, length, nodes, new, dim):
    c = Case(form, dtype, 1, nodes, 4, 1, dim, 16, [length], size=0.3, new=new)
    got, _ = c.call()
    got, eps = got[0].double(), torch.finfo(c.t).eps / 2
    ids = c.table[0].long().cuda()
    keys, values, parts = (x[ids].flatten(0, 1)[:length, 0].cuda() for x in _pools(c))
    sees = torch.ones(nodes, length, dtype=torch.bool, device="cuda")
    if new:
        keys, values, parts = (torch.cat([a, b[0, :, 0].double().cuda()]) for a, b in ((keys, c.k_new), (values, c.v_new), (parts, c.v_new.abs())))
        sees = torch.cat([sees, c.sees[0].cuda()], 1)
    q = c.q[0].double().cuda()
    for h in range(4):
        x = (q[:, h] @ keys.t().contiguous() * c.scale).masked_fill(~sees, -math.inf)
        p = torch.softmax(x, 1)
        want = p @ values
        # A score is a sum of `dim` products and an offset in 32 bits, an exponent's error is a weight's relative one, in numerator and denominator; what two roundings leave of a weight is 2^-8 of 2^-8 where it is
        # kept in bfloat16 (of the cached tokens whatever the type is), 2^-11 of 2^-11 in float16; sums are in 32 bits and the result is rounded once.
        size = q[:, h].abs() @ keys.abs().t().contiguous() * c.scale
        score = 2.0 ** -23 * (dim + 8) * 2 * size.max() + 2.0 ** -20      # (codes and offset may cancel: twice their sum, at most)
        some = 2.0 ** -16 + 2 * score + 2 * (length + nodes + 8) * 2.0 ** -24
        bound = some * (p @ parts) + eps * want.abs() + torch.finfo(c.t).smallest_normal * eps
        assert ((got[:, h] - want).abs() <= bound).all(), ((got[:, h] - want).abs() / bound).max()


def _pools(c):
    """Keys, values and how large codes times scales of the values get, and the offset beside them."""
    k, v = (decoded(p[1].cpu(), s[1].cpu(), c.form) for p, s in ((c.cache.k, c.cache.k_scales), (c.cache.v, c.cache.v_scales)))
    s = c.cache.v_scales[1].cpu().double()
    return [k.cuda(), v.cuda(), ((s[..., 1:].abs() + s[..., :1] * 7.5).expand(v.shape) if c.form == "int4" else v.abs()).cuda()]
