"""Both sides of the sizes at which the adapted layer, its gradients and the
token loss change their way of working, and scales at the ends of their range,
against 64-bit plain implementations."""
from __future__ import annotations

import pytest
import torch

from tests import adapt_ref as ref
from tests.test_gpu_adapt import S_G, _bf, _check_grad, _check_linear, _close, _gen, _low, _problem
from tests.test_gpu_loss import _check_grad as _check_loss_grad, _check_loss, _problem as _loss_problem

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


# Tokens around 16, 64, 128 and 1024; rows of an odd number of 16s; few outputs
# (split k) and many (none); adapters small enough for one launch and too large
# for it; products of 128 x 128, 256 x 128 and 256 x 256 tiles.
@pytest.mark.parametrize("T,n,m,count,rank,how", [
    (2, 2064, 3, 2, 256, "each"), (15, 1008, 700, 200, 8, "each"), (31, 4112, 33, 2, 16, "runs"),
    (48, 336, 2500, 3, 16, "each"), (63, 16, 5000, 1, 8, "runs"), (66, 1008, 700, 2, 8, "each"),
    (127, 528, 33, 9, 40, "runs"), (129, 4112, 17, 1, 16, "each"), (255, 176, 1030, 33, 24, "each"),
    (640, 2064, 130, 3, 136, "runs"), (1023, 144, 520, 4, 8, "each"), (1024, 1040, 64, 2, 256, "runs"),
    (1025, 144, 520, 4, 8, "each"), (1025, 80, 100, 0, 0, ""), (2100, 1040, 300, 3, 40, "runs"),
    (3000, 272, 1500, 2, 16, "each"), (1100, 48, 7000, 2, 8, "runs")])
def test_linear_on_both_sides_of_every_change(hs, T, n, m, count, rank, how):
    _check_linear(hs, _problem(T, n, m, count, rank, seed=3 * T + n, how=how))


@pytest.mark.parametrize("T,n,m,count,rank,how", [
    (16, 64, 3, 40, 256, "each"), (129, 1040, 33, 1, 8, "runs"), (700, 2064, 528, 2, 136, "runs"),
    (1024, 48, 1040, 3, 40, "each"), (1500, 528, 2000, 2, 16, "runs"), (3000, 1040, 96, 20, 72, "each")])
def test_gradients_on_both_sides_of_every_change(hs, T, n, m, count, rank, how):
    p = _problem(T, n, m, count, rank, seed=5 * T + n, how=how)
    _check_grad(hs, p, _bf((T, m), 1.0, _gen(T + 1)))


@pytest.mark.parametrize("s_g", [2.0 ** -100, 2.0 ** -20 * 1.9999, 0.75, 2.0 ** 20])
@pytest.mark.parametrize("T", [3, 90, 1200])
def test_global_scales_from_tiny_to_large(hs, s_g, T):
    """s_g = f 2^e enters as an exact 2^e in the weights and f on the sum."""
    p = _problem(T, 144, 50, 2, 8, seed=T)
    p["B"] *= s_g / S_G
    W = ref.weights(s_g, p["codes"], p["packed"])
    want, size = ref.linear(p["X"], W, **_low(p))
    got = hs.adapted_linear(p["X"], s_g, p["codes"], p["packed"], **_low(p))
    torch.cuda.synchronize()
    _close(got, want, size, "Y")


@pytest.mark.parametrize("T", [5, 200, 1300])
def test_groups_of_scale_zero_and_subnormal_scales(hs, T):
    p = _problem(T, 48, 40, 1, 8, seed=2)
    p["codes"] = torch.randint(0, 8, p["codes"].shape, generator=_gen(4), dtype=torch.int32).to(torch.uint8).to(DEV)
    p["codes"][0], p["codes"][1, 0], p["codes"][2, 0] = 0, 126, 0
    _check_linear(hs, p)


# Two bf16 parts up to 64 tokens, one above.
@pytest.mark.parametrize("T,d,V", [(3, 128, 101), (64, 96, 700), (65, 96, 700), (600, 208, 1500)])
def test_loss_gradients_of_equal_weights_are_rounded_once(hs, T, d, V):
    """A mean's weights of 1 / n.  Rounding to bf16 errs by at most 2^-8 / sqrt(3)
    of the norm (uniform in a unit of 2^-7 of a value's power of two); with g in
    one part, the softmax's share of it, below the target's, is rounded too."""
    X, W, target, _ = _loss_problem(T, d, V, seed=T)
    ok = (target >= 0) & (target < V)
    weight = ok.float() / ok.sum()
    _, lse = hs.token_loss(X, W, target)
    got = hs.token_loss_grad(X, W, target, lse, weight)
    torch.cuda.synchronize()
    want, _ = ref.loss_grad(X, W, target, weight)
    for name, a, b in zip(("dX", "dW"), got, want):
        error = ((a.cpu().double() - b).norm() / b.norm()).item()
        assert error <= 2.0 ** -8 / 3 ** 0.5 * (1.02 if T <= 64 else 1.2), (name, error)


@pytest.mark.parametrize("T", [7, 300])
def test_loss_gradients_of_weights_that_differ_widely(hs, T):
    """Each row of dX is as exact as its own weight allows, whatever the
    largest: bf16 holds 2^-60 of it as well as it."""
    d, V = 64, 200
    X, W, target, _ = _loss_problem(T, d, V, seed=6)
    target = torch.randint(0, V, (T,), generator=_gen(1)).to(DEV)
    weight = torch.ldexp(torch.ones(T), -torch.arange(T) % 61).to(DEV) * 1.1
    weight[1::2] *= -1.0
    _, lse = hs.token_loss(X, W, target)
    dX, dW = hs.token_loss_grad(X, W, target, lse, weight)
    torch.cuda.synchronize()
    (want, want_dW), (size, size_dW) = ref.loss_grad(X, W, target, weight)
    logit = 2.0 ** -15 * (X.cpu().double().abs() @ W.cpu().double().abs().t()).max().item()
    for a, b, s in ((dX, want, size), (dW, want_dW, size_dW)):
        assert ((a.cpu().double() - b).abs() <= 2.0 ** -8 * b.abs() + (2.0 ** -8 + logit + 2.0 ** -15) * s).all()


def test_a_weight_that_is_not_finite_reaches_only_its_row_of_dx(hs):
    T, d, V = 100, 48, 130
    X, W, target, weight = _loss_problem(T, d, V, seed=8)
    target[:5] = 1
    weight[:5] = 0.25
    _, lse = hs.token_loss(X, W, target)
    plain, _ = hs.token_loss_grad(X, W, target, lse, weight, need_dW=False)
    weight[0], weight[3] = float("nan"), float("inf")
    got, _ = hs.token_loss_grad(X, W, target, lse, weight, need_dW=False)
    torch.cuda.synchronize()
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    keep[[0, 3]] = False
    assert torch.equal(got[keep], plain[keep])
    assert not torch.isfinite(got[[0, 3]].float()).all(1).any()


@pytest.mark.parametrize("T,d,V", [(1, 4096, 3), (20, 8192, 500), (64, 2064, 1001), (130, 4112, 258), (3, 1024, 9001)])
def test_loss_of_few_tokens_and_words_of_many_k(hs, T, d, V):
    X, W, target, weight = _loss_problem(T, d, V, seed=T + V)
    _, lse = _check_loss(hs, X, W, target)
    _check_loss_grad(hs, X, W, target, weight, lse)


def test_loss_rows_that_are_not_finite_stay_alone(hs):
    T, d, V = 20, 4096, 300
    X, W, target, weight = _loss_problem(T, d, V, seed=1)
    target[7], target[8] = -100, 5
    loss, lse = hs.token_loss(X, W, target)
    X = X.clone()
    X[7], X[8] = float("nan"), float("nan")
    got, got_lse = hs.token_loss(X, W, target)
    torch.cuda.synchronize()
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    keep[[7, 8]] = False
    assert torch.equal(got[keep], loss[keep]) and torch.equal(got_lse[keep], lse[keep])
    assert got[7] == 0 and got[8].isnan() and got_lse[[7, 8]].isnan().all()
