"""CPU: a cache of the other kind is refused, whichever way a call goes, and never looked at as if it were of the kind that the call takes."""
import pytest

import paper_2508_06041_amd as dp
import test_step_devices as step
import test_token_devices as token
from test_step_devices import made  # noqa: F401
from test_token_devices import made as made_of_tokens  # noqa: F401


class Neither:
    """What the native part looks at of a cache, and no cache."""

    def __init__(self, cache):
        self.k, self.address, self.batch, self.device = cache.k, cache.address, cache.batch, cache.device


@pytest.mark.parametrize("f", ["dpllm_quantized_append", "dpllm_quantized_read", "dpllm_quantized_attention"])
@pytest.mark.parametrize("wrong", [token.cache, lambda: Neither(step.cache())])
def test_not_a_quantized_cache(made, f, wrong):  # noqa: F811
    for args in step.ways(f, step.CALLS[f]()):
        with pytest.raises(dp.DpllmError, match="QuantizedCache"):
            getattr(dp, f)(**dict(args, cache=wrong()))
    assert made == []


@pytest.mark.parametrize("f", ["dpllm_tree_attention", "dpllm_cache_append"])
@pytest.mark.parametrize("wrong", [step.cache, lambda: step.cache("int4"), lambda: Neither(token.cache())])
def test_not_a_cache_of_numbers(made_of_tokens, f, wrong):  # noqa: F811
    for args in token.ways(f, token.CALLS[f]()):
        with pytest.raises(dp.DpllmError, match="has to be a Cache"):
            getattr(dp, f)(**dict(args, cache=wrong()))
    assert made_of_tokens == []


def test_caches_of_a_derived_class(made):  # noqa: F811
    class Own(dp.QuantizedCache):
        pass
    args = step.append_args()
    c = args["cache"]
    own = Own(c.k, c.v, c.k_scales, c.v_scales, c.format, c.table)
    dp.dpllm_quantized_append(**dict(args, cache=own))
    dp.dpllm_quantized_append(**dict(args, cache=own, count=None))
    assert step.names(made) == ["dpllm_quantized_append"] * 2
