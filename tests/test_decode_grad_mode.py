"""Gradients that the calls of a decode step would lose (CPU only,
'meta' tensors): the calls record no graph, so where one would be expected they
refuse, whichever tensor asks for it."""
import pytest
import torch

from paper_2608_28113_amd import ops
from tests.test_decode_abi import CASES
from tests.test_front_end import Reached, fake_gpu  # noqa: F401

FLOATS = ([("route_tokens", a) for a in ("logits", "weight")]
          + [("expert_layer", a) for a in ("X", "weight", "gs", "us", "ds", "Y")]
          + [("adjust_logits", a) for a in ("logits", "repetition", "frequency", "presence", "bias", "out")])


@pytest.mark.parametrize("fn,arg", FLOATS)
def test_every_tensor_that_requires_a_gradient_is_refused(fake_gpu, fn, arg):  # noqa: F811
    f, good, _ = CASES[fn]
    kwargs = good()
    kwargs[arg] = kwargs[arg].detach().requires_grad_()
    with pytest.raises(ValueError, match="no_grad"):
        f(**kwargs)
    with torch.no_grad(), pytest.raises(Reached):
        f(**kwargs)


def test_matrices_may_come_as_any_three(fake_gpu):  # noqa: F811
    _, good, _ = CASES["expert_layer"]
    a = good()
    gate, up, down = (tuple(a[m + f] for f in "scp") for m in "gud")
    with pytest.raises(Reached):
        ops.expert_layer(a["X"], a["expert"], a["weight"], gate, dict(zip("abc", up)).values(), iter(down), stream=0)
