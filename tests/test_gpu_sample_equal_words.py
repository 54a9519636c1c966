"""Draws among words that are all equally likely: sums are whole numbers, and so is every answer, also where the uniform number or top-p lies on a border."""
import math
import random

import pytest
import torch

import paper_2508_06041_amd as dp
from test_gpu_sample import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v", [(1, 40), (2, 2), (1000, 1000), (1024, 5000), (1025, 5000), (2048, 2048), (4096, 9999), (32768, 50000), (30000, 128256), (65536, 65536)])
@pytest.mark.parametrize("top", [0.0, 3.25, -7.0, math.inf])
def test_equal_words(dtype, n, v, top):
    rng = random.Random(n + v)
    settings = [(u, p, k, t) for u in (0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, rng.randrange(2 ** 24) * 2.0 ** -24, rng.randrange(2 ** 9) * 2.0 ** -9)
                for p, k in ((None, None), (0.5, None), (0.125, None), (0.75, n - n // 3), (1.0, n // 2 + 1), (1 - 2.0 ** -24, None)) for t in (1.0, 0.37)]
    x = torch.full((len(settings), v), -math.inf)
    places = []
    for i in range(len(settings)):
        at = sorted(rng.sample(range(v), n))
        x[i, at] = top
        places.append(at)

    def on(values, dtype=torch.float32):
        return torch.tensor(values, dtype=dtype, device="cuda")
    kept = torch.zeros(len(settings), dtype=torch.int32, device="cuda")
    words = dp.dpllm_sample(x.to(TYPES[dtype]).cuda(), on([s[0] for s in settings]), on([s[3] for s in settings]), top_k=on([s[2] or 0 for s in settings], torch.int32),
                            top_p=on([1.0 if s[1] is None else s[1] for s in settings]), kept=kept)
    want = []
    for (u, p, k, _), at in zip(settings, places):
        m = min(n, k or n)
        m = m if p is None or p >= 1 else max(1, math.ceil(p * m))      # i of them are in front of the i-th, less than p m
        want.append((m, at[min(math.floor(u * m), m - 1)]))
    assert list(zip(kept.tolist(), words.tolist())) == want
