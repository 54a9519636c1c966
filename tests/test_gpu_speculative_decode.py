"""The calls around the linears together, as examples/speculative_decode.py uses them."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nodes", [2, 6])
def test_drafts_change_nothing_but_the_number_of_steps(nodes):
    """With the best token taken, what stands is what the target alone decodes.  (A row's products may be added up in another order beside more rows, which
    would show where two logits are that close; they are not on this path.)"""
    import speculative_decode as s
    plain = s.Decoder()
    want, steps = plain.decode(1, 60, 0.0, 1)
    assert steps == 60 and plain.lens.item() == 60
    fast = s.Decoder()
    got, steps = fast.decode(1, 60, 0.0, nodes)
    assert got[:60] == want
    assert steps < 60 and fast.lens.item() == len(got)
    # the caches agree: what was refused never entered
    n = 59
    for a, b in ((plain.k, fast.k), (plain.v, fast.v)):
        rows = [x[:, p.cache.table[0].long()].flatten(1, 2)[:, :n].float() for x, p in ((a, plain), (b, fast))]
        assert (rows[0] - rows[1]).abs().max() < 0.05 * rows[0].abs().max()


def test_with_a_temperature():
    import speculative_decode as s
    d = s.Decoder()
    out, steps = d.decode(1, 80, 0.7)
    assert len(out) >= 80 and all(0 <= w < s.WORDS for w in out) and d.lens.item() == len(out)
    assert steps <= len(out)
    assert torch.isfinite(d.k.float()).all() and torch.isfinite(d.v.float()).all()
