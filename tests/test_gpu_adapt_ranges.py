"""Global scales at the ends of what is accepted, and rows so far apart that
they pass 32 bits of bytes, against 64 bits and against rows side by side."""
from __future__ import annotations

import pytest
import torch

from tests import adapt_ref as ref
from tests.test_gpu_adapt import DEV, S_G, _bf, _close, _gen, _low, _problem
from tests.test_gpu_loss import _problem as _loss_problem

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


SCALES = [2.0 ** -117, 2.0 ** -110 * 1.3, 2.0 ** 100, 2.0 ** 116 * 1.9, 2.0 ** 117, 2.0 ** 118 * 1.1, 2.0 ** 119 * 0.99]


@pytest.mark.parametrize("s_g", SCALES)
@pytest.mark.parametrize("T", [3, 90, 1200])
def test_layer_and_gradients_at_any_accepted_scale(hs, s_g, T):
    """Values of X, dY and B that keep every result of the formulas, and each of
    its terms, within bf16's range."""
    n, m = 144, 50
    x = 2.0 ** -60 if s_g > 1.0 else 1.0
    p = _problem(T, n, m, 2, 8, seed=T)
    p["X"] *= x
    p["B"] *= s_g / S_G * 2.0 ** -8
    W = ref.weights(s_g, p["codes"], p["packed"])
    want, size = ref.linear(p["X"], W, **_low(p))
    _close(hs.adapted_linear(p["X"], s_g, p["codes"], p["packed"], **_low(p)), want, size, "Y")
    dY = _bf((T, m), x, _gen(T))
    q, scale = hs.pack_activations(p["X"])
    want, size = ref.linear_grad(dY, hs.unpack_activations(q, scale), W, **_low(p))
    got = hs.adapted_linear_grad(dY, q, scale, s_g, p["codes"], p["packed"], **_low(p))
    torch.cuda.synchronize()
    # below its smallest normal value bf16 rounds to multiples of 2^-133
    for name, a, b, s in zip(("dX", "dA", "dB"), got, want, size):
        _close(a, b, s + 2.0 ** -118, name)


@pytest.fixture(scope="module")
def far():
    """Two buffers whose rows are 4 MB apart, 4.6 GB each."""
    return [torch.zeros((1100, 1 << 21), dtype=torch.bfloat16, device=DEV) for _ in range(2)]


@pytest.mark.parametrize("T", [1, 40, 300, 1024, 1100])
def test_layer_reads_and_writes_rows_that_pass_32_bits(hs, far, T):
    n, m = 64, 80
    p = _problem(T, n, m, 3, 16, seed=T)
    X, Y = far[0][:T, 128:128 + n], far[1][:T, 4096:4096 + m]
    X.copy_(p["X"])
    want = hs.adapted_linear(p["X"], S_G, p["codes"], p["packed"], **_low(p))
    hs.adapted_linear(X, S_G, p["codes"], p["packed"], **_low(p), Y=Y)
    torch.cuda.synchronize()
    assert torch.equal(Y, want)


def test_checkpoint_and_gradients_read_and_write_rows_that_pass_32_bits(hs, far):
    T, n, m = 1100, 64, 80
    p = _problem(T, n, m, 3, 16, seed=1)
    X, dY, back, dX = far[0][:, 128:128 + n], far[0][:, 8192:8192 + m], far[1][:, 16:16 + n], far[1][:, 520:520 + n]
    X.copy_(p["X"])
    dY.copy_(_bf((T, m), 1.0, _gen(2)))
    q, scale = hs.pack_activations(p["X"])
    got_q, got_scale = hs.pack_activations(X)
    hs.unpack_activations(q, scale, X=back)
    args = (q, scale, S_G, p["codes"], p["packed"])
    want = hs.adapted_linear_grad(dY.contiguous(), *args, **_low(p))
    got = hs.adapted_linear_grad(dY, *args, **_low(p), dX=dX)
    torch.cuda.synchronize()
    assert torch.equal(got_q, q) and torch.equal(got_scale, scale)
    assert torch.equal(back, hs.unpack_activations(q, scale))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_loss_and_gradient_read_and_write_rows_that_pass_32_bits(hs, far):
    T, d, V = 1100, 64, 300
    X, W, target, weight = _loss_problem(T, d, V, seed=2)
    wide, dX = far[0][:, 64:64 + d], far[1][:, 8:8 + d]
    wide.copy_(X)
    loss, lse = hs.token_loss(X, W, target)
    want = loss, lse, *hs.token_loss_grad(X, W, target, lse, weight)
    loss, lse = hs.token_loss(wide, W, target)
    got = loss, lse, *hs.token_loss_grad(wide, W, target, lse, weight, dX=dX)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
