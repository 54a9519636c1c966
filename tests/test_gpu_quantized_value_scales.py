"""Attention over a quantised cache in which a token's values are many times the others': those that it hardly counts for keep what they have."""
import pytest
import torch

import paper_2508_06041_amd as dp
from test_gpu_quantized_attention import Case, ints, normal
from test_gpu_quantized_cache import FORMS
from test_gpu_tree_attention import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nodes,heads,dim,lens", [(1, 8, 128, [200]), (3, 4, 64, [333, 70]), (1, 8, 256, [90]), (9, 8, 96, [100]), (20, 8, 128, [500]), (40, 8, 64, [300])])
@pytest.mark.parametrize("size", [12, 30, 60])
def test_a_token_of_large_values(form, dtype, nodes, heads, dim, lens, size):
    """Queries of the first half of the heads of a group see it with a weight of e^-50 or less, those of the others see hardly anything else."""
    c = Case(form, dtype, len(lens), nodes, heads, 2, dim, 16, lens)
    sign = torch.where(torch.arange(heads) % (heads // 2) < heads // 4, 1.0, -1.0)[:, None]
    c.q = (normal(*c.q.shape, seed=7).abs() * sign).to(c.t)
    k = torch.full((len(lens), 1, 2, dim), -20.0)
    v = normal(len(lens), 1, 2, dim, seed=8) * 2.0 ** size
    for at in (3, 66):
        dp.dpllm_quantized_append(c.cache, ints([at] * len(lens)), k.cuda(), v.cuda(), layer=1)
    got, _ = c.call()
    want, _ = c.plain()
    # Beside a token that takes all, weights (and weights times scales, for codes up to 448) below the smallest normal float may be lost.
    most = max(v.abs().max().item(), c.v_new.double().abs().max().item(), 8.0)
    lost = (lens[0] + nodes) * 2.0 ** -126 * (448 + most)
    got, top = got.double().cpu(), torch.finfo(c.t).max
    held = want.abs() < top            # the largest values are past those of float16
    assert ((got - want).abs() <= c.bound + lost)[held].all()
    assert (got.abs() >= top * (1 - 2.0 ** -8))[~held].all() and (got * want >= 0)[~held].all()
