"""Gradients and tangents that the calls of a decode step would lose (CPU only,
'meta' tensors): the calls record no graph, so where one would be expected they
refuse, whichever tensor asks for it."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2608_28113_amd import ops
from tests import test_adapt_abi
from tests.test_decode_abi import CASES
from tests.test_front_end import Reached, fake_gpu  # noqa: F401

FLOATS = ([("route_tokens", a) for a in ("logits", "weight")]
          + [("expert_layer", a) for a in ("X", "weight", "gs", "us", "ds", "Y")]
          + [("adjust_logits", a) for a in ("logits", "repetition", "frequency", "presence", "bias", "out")])
EARLIER = [("adapted_linear", a) for a in ("X", "A", "B", "alpha")] + [("token_loss", a) for a in ("X", "W")]


@pytest.mark.parametrize("fn,arg", FLOATS)
def test_every_tensor_that_requires_a_gradient_is_refused(fake_gpu, fn, arg):  # noqa: F811
    f, good, _ = CASES[fn]
    kwargs = good()
    kwargs[arg] = kwargs[arg].detach().requires_grad_()
    with pytest.raises(ValueError, match="no_grad"):
        f(**kwargs)
    with torch.no_grad(), pytest.raises(Reached):
        f(**kwargs)


@pytest.mark.parametrize("fn,arg", FLOATS + EARLIER)
@pytest.mark.parametrize("mode", [torch.enable_grad, torch.no_grad])
def test_a_tangent_is_refused(fake_gpu, fn, arg, mode):  # noqa: F811
    """torch carries tangents forward under no_grad too."""
    if (fn, arg) in FLOATS:
        f, good, _ = CASES[fn]
        kwargs = good()
    else:
        f, good, _ = test_adapt_abi.CASES[fn]
        kwargs = dict(good(), stream=0)
    with forward_ad.dual_level(), mode():
        with pytest.raises(Reached):  # a level alone loses nothing
            f(**kwargs)
        kwargs[arg] = forward_ad.make_dual(kwargs[arg].detach(), torch.ones_like(kwargs[arg]))
        with pytest.raises(ValueError, match="tangent"):
            f(**kwargs)


@pytest.mark.parametrize("fn,arg", [("expert_layer", "X"), ("adjust_logits", "logits"), ("adapted_linear", "X")])
def test_inside_an_autograd_function_tangents_are_its_own(fake_gpu, fn, arg):  # noqa: F811
    f, good, _ = (CASES if fn in CASES else test_adapt_abi.CASES)[fn]
    kwargs = good() if fn in CASES else dict(good(), stream=0)

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, t):
            kwargs[arg] = t
            return f(**kwargs)

        @staticmethod
        def jvp(ctx, tangent):
            return tangent

    with forward_ad.dual_level():
        dual = forward_ad.make_dual(kwargs[arg].detach(), torch.ones_like(kwargs[arg]))
        with pytest.raises(Reached):
            Layer.apply(dual)


def test_matrices_may_come_as_any_three(fake_gpu):  # noqa: F811
    _, good, _ = CASES["expert_layer"]
    a = good()
    gate, up, down = (tuple(a[m + f] for f in "scp") for m in "gud")
    with pytest.raises(Reached):
        ops.expert_layer(a["X"], a["expert"], a["weight"], gate, dict(zip("abc", up)).values(), iter(down), stream=0)


@pytest.mark.parametrize("arg", ["repetition", "frequency", "presence", "bias", "out"])
def test_numbers_in_place_of_tensors_are_refused(fake_gpu, arg):  # noqa: F811
    f, good, _ = CASES["adjust_logits"]
    with pytest.raises(ValueError):
        f(**{**good(), arg: 1.5})
