"""Draws at the very start of the running sum, where the first chunks of a row hold next to nothing: a token is found all the same."""
import math

import pytest
import torch

import paper_2508_06041_amd as dp
from test_gpu_verify import TYPES, compare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap", [5.0, 6.4, 6.75, 6.95, 7.3, 7.6])
@pytest.mark.parametrize("named", [True, False])
def test_chunks_far_below_the_largest_logit(dtype, gap, named):
    """At a temperature of 0.01 the first words have e^-500 to e^-760 of the last one's weight: the first is drawn where that is above 1e-280, else the last."""
    v = 20000
    logits = torch.full((1, 1, v), -gap).to(TYPES[dtype])
    logits[..., v - 1] = 0.0
    weight = logits[0, 0, 0].double().item() / 0.01
    words = dp.dpllm_verify(logits.cuda(), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, device="cuda"), torch.full((1,), 0.01, device="cuda"),
                            draft=None if named else logits.cuda())[2]
    assert words.item() == (0 if weight > math.log(1e-280) else v - 1)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_chunk_whose_words_were_all_refused(dtype):
    """Three words have a probability; two of one chunk are named and refused, and the third is what is left."""
    b, v = 64, 20000
    g = torch.Generator().manual_seed(5)
    logits = torch.full((b, 3, v), -math.inf)
    logits[:, :, [3, 10, 15000]] = torch.rand(b, 3, 3, generator=g) * 0.5
    tokens = torch.tensor([[0, 3, 10]] * b, dtype=torch.int32)
    parents = torch.tensor([[-1, 0, 0]] * b, dtype=torch.int32)
    uniforms = torch.full((b, 3), 1.0 - 2.0 ** -24)
    uniforms[:, 0] = 0.0
    lengths = compare(logits.to(TYPES[dtype]).cuda(), tokens.cuda(), parents.cuda(), uniforms.cuda(), torch.full((b,), 0.8, device="cuda"), None)
    assert lengths == [1] * b


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap", [6.4, 6.75, 6.95, 7.6])
def test_beside_a_draft_without_a_number(dtype, gap):
    """The same behind a child that is no word, with a draft row that takes nothing away."""
    v = 20000
    logits = torch.full((1, 2, v), -gap).to(TYPES[dtype])
    logits[..., v - 1] = 0.0
    weight = logits[0, 0, 0].double().item() / 0.01
    tokens = torch.full((1, 2), -1, dtype=torch.int32, device="cuda")
    words = dp.dpllm_verify(logits.cuda(), tokens, torch.zeros(1, 2, device="cuda"), torch.full((1,), 0.01, device="cuda"),
                            draft=torch.full_like(logits, -math.inf).cuda())[2]
    assert words.tolist() == [[0 if weight > math.log(1e-280) else v - 1, -1]]
