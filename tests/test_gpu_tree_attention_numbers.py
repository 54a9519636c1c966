"""Attention of drafted tokens where queries, seen keys or scores are no ordinary numbers, against the formula in 64 bits."""
import math

import pytest
import torch

from test_gpu_tree_attention import TYPES, Case, words

pytestmark = pytest.mark.gpu

# nodes, heads, kv heads: one row to a kv head, a tile of 16 rows that is full, one of 32, and the kernels for many rows
ROWS = [(1, 2, 2), (1, 16, 1), (4, 8, 1), (9, 8, 2), (70, 4, 2)]
LENGTHS = [40, 3000]      # in one part and in several


def check(c, **kw):
    """As Case.check(), and NaN are where the formula has them, in the rows and in lse."""
    out, lse = (x.double().cpu() for x in c.run(**kw))
    want, want_lse = c.plain()
    assert torch.equal(out.isnan(), want.isnan()) and torch.equal(lse.isnan(), want_lse.isnan())
    some = ~want.isnan()
    assert ((out - want).abs() <= c.bound)[some].all()
    some, none = ~want_lse.isnan() & (want_lse != -math.inf), want_lse == -math.inf
    assert torch.equal(lse == -math.inf, none) and ((lse - want_lse).abs() <= c.lse_bound)[some].all()
    return want_lse


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", LENGTHS)
@pytest.mark.parametrize("nodes,heads,kv", ROWS)
def test_queries_that_are_no_numbers(dtype, nodes, heads, kv, length):
    """A NaN in a query, or an infinity that meets keys of both signs, makes its row NaN and no other one, however the work is split."""
    c = Case(dtype, 2, nodes, heads, kv, 128, 16, [length, 5], mask="tree", seed=nodes)
    c.q[0, nodes - 1, 0, 5] = math.nan
    if heads > 2:
        c.q[0, 0, heads - 1, 127], c.q[1, 0, 2, 0] = math.inf, math.nan
        c.q[0, 0, heads - 1, 126] = math.inf
    lse = check(c)
    assert lse.isnan().sum() == (1 if heads == 2 else 3)
    for max_len in (0, 100000):
        check(c, max_len=max_len)
    c.q[:] = math.nan
    assert check(c).isnan().all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", LENGTHS)
@pytest.mark.parametrize("nodes,heads,kv", ROWS)
def test_seen_keys_that_are_no_numbers(dtype, nodes, heads, kv, length):
    """A NaN in a key makes the rows that see it NaN."""
    c = Case(dtype, 2, nodes, heads, kv, 64, 16, [length, 5], mask="any", seed=nodes)
    c.sees[:, :, nodes - 1] = False
    c.sees[0, ::2, nodes - 1] = True
    c.mask = words(c.sees)
    c.k_new[0, nodes - 1, 0, 3] = math.nan
    lse = check(c)
    assert torch.equal(lse[0, :, 0].isnan(), c.sees[0, :, nodes - 1]) and not lse[1].isnan().any()
    at = c.table[1, 0].item()
    c.k[0, at, 4, kv - 1, 0] = math.nan      # the last token of the second sequence
    lse = check(c)
    assert lse[1, :, heads - 1].isnan().all()
    if length > 1000:                        # among a thousand others, in one of the middle parts
        c.k[0, c.table[0, 100].item(), 7] = math.nan
        assert check(c)[0].isnan().all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("length", LENGTHS)
@pytest.mark.parametrize("nodes,heads,kv", ROWS)
@pytest.mark.parametrize("value", [1e5, -3e6, 1e9, -1e12, 1e20, -1e36, 1e38])
def test_scores_far_from_zero(dtype, length, nodes, heads, kv, value):
    """The same score for all tokens, another one in every row: all weights are equal.  Then one token further from zero: it has all of the weight, or none."""
    c = Case(dtype, 1, nodes, heads, kv, 64, 16, [length], new=False, scale=value)
    c.q[:], c.k[:] = 0.0, 0.0
    size = 1 + torch.arange(nodes * heads).reshape(nodes, heads) % 64 / 64      # good in either type
    c.q[0, :, :, 0] = size.to(c.t)
    c.k[..., 0] = 1.0
    values = c.v[0, c.table[0].long()].flatten(0, 1)[:length].double().repeat_interleave(heads // kv, 1)      # [token][head][d]
    odd = length // 3
    for alone in (False, True):
        if alone:
            c.k[0, c.table[0, odd // 16], odd % 16, :, 0] = 1.5
        out, lse = (x.double().cpu() for x in c.run())
        some = values if not alone else values[odd:odd + 1] if value > 0 else torch.cat([values[:odd], values[odd + 1:]])
        want = some.mean(0)
        # equal weights are rounded alike, half a step; sums in 32 bits, one rounding of the result
        eps = torch.finfo(c.t).eps / 2
        bound = (eps + (length + 4) * 2.0 ** -24) * some.abs().mean(0) + eps * want.abs() + 2.0 ** -24
        assert ((out[0] - want).abs() <= bound).all()
        top = size.double() * value * (1.5 if alone and value > 0 else 1.0)
        assert ((lse[0] - top).abs() <= 2.0 ** -21 * top.abs() + math.log(length) + 1).all()


@pytest.mark.parametrize("length", LENGTHS)
@pytest.mark.parametrize("nodes,heads", [(1, 1), (1, 16), (2, 16), (4, 16), (9, 16)])
@pytest.mark.parametrize("value", [torch.finfo(torch.bfloat16).min, -2e37])
def test_scores_next_to_the_lowest(length, nodes, heads, value):
    """Scores that are all the same, far below zero: all weights are equal, in tiles that are full and in such that are not."""
    c = Case("bf16", 1, nodes, heads, 1, 64, 16, [length], new=False, scale=1.0)
    c.q[:], c.k[:] = 0.0, 0.0
    c.q[..., 0] = 1.0
    c.k[..., 0] = value
    out, lse = c.run()
    values = c.v[0, c.table[0].long(), :, 0].flatten(0, 1)[:length].double()
    want = values.mean(0)
    # the weights are powers of two up to the last bit of a float; sums in 32 bits, one rounding of the result
    bound = (length + 4) * 2.0 ** -24 * values.abs().mean(0) + 2.0 ** -8 * want.abs() + 2.0 ** -24
    assert ((out.double().cpu() - want).abs() <= bound).all()
    assert (lse / c.k[0, 0, 0, 0, 0].item() - 1).abs().max() <= 2.0 ** -20
