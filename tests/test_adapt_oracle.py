"""The plain gradients that the kernels are compared with, against difference
quotients of the plain forward pass (CPU, float64)."""
import pytest
import torch

from tests import adapt_ref as ref


def _problem(T, n, m, count, rank, seed):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    adapter = torch.randint(-1, count + 1, (T,), generator=g, dtype=torch.int32)
    return rand(T, m), rand(T, n), rand(m, n), rand(count, rank, n), rand(count, m, rank), rand(count), adapter


@pytest.mark.parametrize("T,n,m,count,rank", [(1, 16, 1, 1, 8), (7, 32, 5, 3, 8), (20, 16, 11, 2, 16)])
def test_layer_gradients_are_the_differences(T, n, m, count, rank):
    """The layer is linear in X, in A and in B: a difference quotient has no
    error but rounding, 2^-52 of the terms over the step of 1."""
    dY, X, W, A, B, alpha, adapter = _problem(T, n, m, count, rank, seed=T)
    (dX, dA, dB), size = ref.linear_grad(dY, X, W, A, B, alpha, adapter)

    def total(X, A, B):
        return (ref.linear(X, W, A, B, alpha, adapter)[0] * dY).sum().item()

    g = torch.Generator().manual_seed(5)
    for k, (grad, s) in enumerate(zip((dX, dA, dB), size)):
        D = torch.randn(grad.shape, generator=g, dtype=torch.float64)
        args = [X, A, B]
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + D, args[k] - D
        quotient = (total(*up) - total(*down)) / 2.0
        terms = (s * (D.abs() + 1.0)).sum().item() + abs(total(*up)) + abs(total(*down))
        assert abs(quotient - (grad * D).sum().item()) <= 1e-11 * terms + 1e-12


@pytest.mark.parametrize("T,d,V", [(1, 4, 1), (6, 5, 9), (12, 8, 40)])
def test_loss_gradients_are_the_differences(T, d, V):
    """Central differences: an error of step^2 / 6 of the third derivative,
    with a step of 1e-4 below 1e-6 of sums of order one to ten."""
    g = torch.Generator().manual_seed(V)
    X = torch.randn((T, d), generator=g, dtype=torch.float64)
    W = torch.randn((V, d), generator=g, dtype=torch.float64)
    target = torch.randint(-1, V + 1, (T,), generator=g)
    weight = torch.randn(T, generator=g, dtype=torch.float64)
    (dX, dW), _ = ref.loss_grad(X, W, target, weight)

    def total(X, W):
        return (ref.loss(X, W, target)[0] * weight).sum().item()

    h = 1e-4
    for k, grad in enumerate((dX, dW)):
        D = torch.randn(grad.shape, generator=g, dtype=torch.float64)
        D /= D.norm()
        up, down = [X, W], [X, W]
        up[k], down[k] = up[k] + h * D, down[k] - h * D
        assert abs((total(*up) - total(*down)) / (2 * h) - (grad * D).sum().item()) <= 1e-6
