"""Verification where the draft is the target: behind a child that can not stand nothing is left of the target beside the draft, and the target's distribution stays."""
import math

import pytest
import torch

from test_gpu_verify import TYPES, compare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v", [64, 1000, 9001])
@pytest.mark.parametrize("alike", [True, False])
def test_a_child_that_can_not_stand(dtype, v, alike):
    """The first children are no words, or words without a probability in either row; then one that stands whatever its uniform, or none."""
    g = torch.Generator().manual_seed(v)
    b, n = 24, 7
    logits = (torch.randn(b, n, v, generator=g) * 2.0).to(TYPES[dtype])
    logits[1] = 0.5                                        # every word alike
    logits[:, :, 3] = -math.inf
    logits = logits.cuda()
    draft = torch.empty(b * n * v + 1, dtype=TYPES[dtype], device="cuda")[0 if alike else 1:][:b * n * v].view(b, n, v)
    draft.copy_(logits)
    tokens = torch.zeros(b, n, dtype=torch.int32)
    tokens[:, 1:] = torch.tensor([-1, 3, 5, 3, v, 5], dtype=torch.int32)
    tokens[::3, 1] = 2 ** 31 - 1
    uniforms = torch.rand(b, n, generator=g)
    uniforms[:, 1:] = 1.0 - 2.0 ** -24
    # the root's third child stands, and under it no child does: the token behind is the target's own draw
    parents = torch.tensor([[-1, 0, 0, 0, 3, 3, 1]] * b, dtype=torch.int32)
    parents[1::2, 3] = -1                                  # no child of the root stands
    lengths = compare(logits, tokens.cuda(), parents.cuda(), uniforms.cuda(), torch.full((b,), 0.9, device="cuda"), draft, siblings=3)
    assert lengths == [2, 1] * (b // 2)


@pytest.mark.parametrize("dtype", TYPES)
def test_something_is_left_beside_rows_that_are_nearly_equal(dtype):
    """One word of a thousand is likelier in the target: behind a refused child it is the only one left."""
    b, n, v = 8, 2, 1000
    g = torch.Generator().manual_seed(3)
    draft = (torch.randn(b, n, v, generator=g) * 2.0).to(TYPES[dtype])
    logits = draft.clone()
    logits[:, 0, 777] += 1.0
    tokens = torch.full((b, n), 3, dtype=torch.int32)
    tokens[1::2, 1] = -1
    uniforms = torch.full((b, n), 1.0 - 2.0 ** -24)
    uniforms[:, 0] = torch.rand(b, generator=g)
    lengths = compare(logits.cuda(), tokens.cuda(), None, uniforms.cuda(), torch.full((b,), 1.1, device="cuda"), draft.cuda())
    assert lengths == [1] * b


@pytest.mark.parametrize("dtype", TYPES)
def test_next_to_nothing_is_left(dtype):
    """Rows that agree on a word of nearly all of the probability: however little the target has more of the others, that is what is left."""
    b, v = 16, 9001
    g = torch.Generator().manual_seed(4)
    logits = torch.rand(b, 3, v, generator=g) * 4.0 - 8.0
    logits[:, :, 100] = 0.0
    draft = logits - 1.0
    draft[:, :, 100] = 0.0
    draft[:, :, 5000:] = logits[:, :, 5000:] + 0.5            # only words before 5000 have something left
    tokens = torch.full((b, 3), -1, dtype=torch.int32)
    tokens[:, 2] = 8000
    tokens[::2, 2] = 7
    uniforms = torch.rand(b, 3, generator=g)
    uniforms[:, 2] = 1.0 - 2.0 ** -24
    parents = torch.tensor([[-1, 0, 0]] * b, dtype=torch.int32)
    temperature = torch.tensor([0.05, 0.06, 0.08, 0.1, 0.12, 0.15, 0.2, 0.4] * 2)
    lengths = compare(logits.to(TYPES[dtype]).cuda(), tokens.cuda(), parents.cuda(), uniforms.cuda(), temperature.cuda(), draft.to(TYPES[dtype]).cuda(), siblings=2)
    assert set(lengths) <= {1, 2}
