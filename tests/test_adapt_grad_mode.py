"""Tensors that require a gradient (CPU only, 'meta' tensors): the calls record
no graph, so where one would be expected they refuse instead of returning a
result that no gradient reaches."""
import pytest
import torch

from paper_2608_28113_amd import ops
from tests.test_adapt_abi import CASES
from tests.test_front_end import Reached, fake_gpu  # noqa: F401

WITH_GRADIENT = [("adapted_linear", a) for a in ("X", "A", "B", "alpha")] + [("token_loss", a) for a in ("X", "W")]


def _given(fn, arg):
    f, good, _ = CASES[fn]
    kwargs = good()
    kwargs[arg] = kwargs[arg].detach().requires_grad_()
    return f, kwargs


@pytest.mark.parametrize("fn,arg", WITH_GRADIENT)
def test_a_graph_that_is_not_recorded_is_refused(fake_gpu, fn, arg):  # noqa: F811
    f, kwargs = _given(fn, arg)
    with pytest.raises(ValueError, match="no_grad"):
        f(**kwargs, stream=0)
    with torch.no_grad(), pytest.raises(Reached):
        f(**kwargs, stream=0)


@pytest.mark.parametrize("fn,arg", WITH_GRADIENT)
def test_inside_an_autograd_function_they_run(fake_gpu, fn, arg):  # noqa: F811
    f, kwargs = _given(fn, arg)

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, t):
            kwargs[arg] = t
            return f(**kwargs, stream=0)

    with pytest.raises(Reached):
        Layer.apply(kwargs[arg])


@pytest.mark.parametrize("fn,arg", [("adapted_linear_grad", a) for a in ("dY", "A", "B", "alpha")]
                         + [("token_loss_grad", a) for a in ("X", "W", "weight")] + [("pack_activations", "X")])
def test_gradients_and_checkpoints_take_parameters(fake_gpu, fn, arg):  # noqa: F811
    """They are the backward pass, or what it keeps; nothing differentiates them."""
    f, kwargs = _given(fn, arg)
    with pytest.raises(Reached):
        f(**kwargs, stream=0)


def test_the_calls_of_the_search_take_parameters(fake_gpu):  # noqa: F811
    """Codes are not differentiable, and a model's weights are parameters."""
    W = torch.nn.Parameter(torch.empty((4, 64), dtype=torch.bfloat16, device="meta"))
    with pytest.raises(Reached):
        ops.search(W, torch.empty(64, device="meta"), 1e-3, window=2, stream=0)
