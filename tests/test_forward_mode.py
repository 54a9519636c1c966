"""CPU: the calls that have a gradient have none in forward mode; a tensor with a tangent is refused rather than taken without it."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2508_06041_amd as dp
import test_step_devices as step
import test_token_devices as token
from test_step_devices import made  # noqa: F401
from test_token_devices import made as made_of_tokens  # noqa: F401


def dual(t):
    return token.on(forward_ad.make_dual(t.as_subclass(torch.Tensor), torch.ones_like(t.as_subclass(torch.Tensor))))


def refused(f, args, names, made):  # noqa: F811
    with forward_ad.dual_level():
        for name in names:
            if name not in args:
                continue
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises(dp.DpllmError, match="forward mode"):
                    getattr(dp, f)(**dict(args, **{name: dual(args[name])}))
                if name != "weights":
                    with torch.set_grad_enabled(grad), pytest.raises(dp.DpllmError, match="forward mode"):
                        getattr(dp, f)(**{k: (dual(v) if k == name else v,) if k in ("x", "grads", "weights", "out") else v for k, v in args.items()})
        assert made == []
        getattr(dp, f)(**args)      # one without a tangent is taken meanwhile
    assert len(made) == 1


@pytest.mark.parametrize("f", ["dpllm_norm_rope", "dpllm_norm_rope_backward"])
def test_norms(made, f):  # noqa: F811
    for args in step.ways(f, step.CALLS[f]()):
        refused(f, args, ("x", "weights", "grads"), made)
        made.clear()


def test_rotary_positions(made_of_tokens):  # noqa: F811
    refused("dpllm_rope", token.rope_args(), ("x",), made_of_tokens)
