"""Zeros of either sign among the values of heads that go into a quantised cache: they are the same value, and what stands beside them is held as it is."""
import pytest
import torch

import paper_2508_06041_amd as dp
from test_gpu_quantized_cache import FORMS, TYPES, check_held, decoded, ints, new_cache

pytestmark = pytest.mark.gpu


def heads(t, dim):
    """Heads with a -0.0 at each place of eight codes: lowest and highest value opposite (an offset of 0), and not; every second value -0.0; nothing but zeros, of one sign and of both."""
    g = torch.Generator().manual_seed(1)
    made = []
    for top, low in ((1.0, -1.0), (1.0, -0.75), (0.0, -2.0), (3.0, 0.0)):
        for place in range(8):
            x = (torch.rand(dim, generator=g) * (top - low) + low) * 0.9
            x[(place + 1) % 8], x[(place + 2) % 8] = top, low
            x[place] = -0.0
            x[8 + place::8][::2] = -0.0
            made.append(x)
    x = torch.rand(dim, generator=g) - 0.5
    x[0], x[2] = 0.5, -0.5
    x[1::2] = -0.0
    made += [x, torch.full((dim,), -0.0), torch.zeros(dim), torch.where(torch.arange(dim) % 3 == 0, -0.0, 0.0)]
    return torch.stack(made).to(t)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [16, 34, 64, 128])
def test_zeros_of_either_sign(form, dtype, dim):
    x = heads(TYPES[dtype], dim)
    n = x.shape[0]
    c = new_cache(form, 1, 3, 16, 1, dim, ints([[2, 0, 1]]))
    for new in (x, -x):
        rows = new.reshape(1, n, 1, dim)
        dp.dpllm_quantized_append(c, ints([0]), rows.cuda(), rows.flip(1).contiguous().cuda())
        for pool, scales, want in ((c.k, c.k_scales, new), (c.v, c.v_scales, new.flip(0))):
            check_held(decoded(pool[0, [2, 0, 1]].flatten(0, 1), scales[0, [2, 0, 1]].flatten(0, 1), form)[:n, 0], want, form)
