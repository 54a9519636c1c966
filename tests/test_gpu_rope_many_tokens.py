"""Rotary positions of more tokens than a grid has workgroups for: those beyond are turned behind the others, by the same workgroups."""
import pytest
import torch

import paper_2508_06041_amd as dp
from test_gpu_rope import check, plain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("tokens,heads,dim", [(2 ** 24 + 2 ** 20 + 3, 1, 8), (2 ** 20 + 777, 130, 4), (2 ** 20 + 5, 33, 64)])
def test_a_grid_is_not_enough(tokens, heads, dim, layout):
    """Sixteen tokens to a workgroup, one in pieces of an element, one in pieces of 16 bytes; a grid has up to 2^20 workgroups."""
    x = torch.randn(1, tokens, heads, dim, generator=torch.Generator("cuda").manual_seed(1), device="cuda", dtype=torch.float16)
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    freqs, _ = dp.dpllm_rope_frequencies(dim)
    got = dp.dpllm_rope(x, pos, freqs, layout=layout)
    turn = 2 ** 24 if heads == 1 else 2 ** 20
    for part in (slice(0, 300), slice(turn - 300, turn + 5), slice(max(turn, tokens - 300), tokens)):
        check(got[:, part], *plain(x[:, part], pos[None, part], freqs, 1.0, layout, False), torch.float16)
    # and no token keeps what it had: the same from a second call over the tokens behind the turn alone
    assert torch.equal(dp.dpllm_rope(x[:, turn - 1000:], pos[turn - 1000:], freqs, layout=layout), got[:, turn - 1000:])
