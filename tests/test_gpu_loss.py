"""The token loss and its gradient against 64-bit plain implementations and
against differences."""
from __future__ import annotations

import math

import pytest
import torch

from tests import adapt_ref as ref

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"
# Logits are fp32 sums of exact products: within (d / 16) 2^-24, at most 2^-15
# here, of the sum of absolute terms; lse and loss as far off as the logits
# that matter, and 2^-20 of fp32 exponentials, logarithm and their sum.
LOGIT = 2.0 ** -15
# g is rounded to bf16 (2^-8 of each term), after a relative error of as much
# as the logits' absolute one; dX and dW are rounded to bf16 once more.  Terms
# below fp32's range are zeros: up to 2^-126 for each of at most 2^14 terms.
ROUND = 2.0 ** -8
RANGE = 2.0 ** -112


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


def _problem(T, d, V, seed, std=2.0):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn((T, d), generator=g).bfloat16().to(DEV)
    W = (torch.randn((V, d), generator=g) * std * d ** -0.5).bfloat16().to(DEV)
    target = torch.randint(0, V, (T,), generator=g)
    target[torch.rand(T, generator=g) < 0.2] = -100
    if T > 4:
        target[2], target[3] = V, V + 12345678901  # past the end: not scored
        target[4] = V - 1
    target = target.to(DEV)
    weight = torch.rand(T, generator=g).to(DEV) / T
    if T > 8:
        weight[6] = 0.0
    return X, W, target, weight


def _check_loss(hs, X, W, target):
    print(f"[loss {tuple(X.shape)} x {W.shape[0]}]", flush=True)
    loss, lse = hs.token_loss(X, W, target)
    torch.cuda.synchronize()
    want, want_lse, logits = ref.loss(X, W, target)
    size = (X.cpu().double().abs() @ W.cpu().double().abs().t()).amax(-1)
    tol = 2 * LOGIT * size + 2.0 ** -20 * (1.0 + logits.abs().amax(-1)) + 2.0 ** -20
    assert ((loss.cpu().double() - want).abs() <= tol).all()
    assert ((lse.cpu().double() - want_lse).abs() <= tol).all()
    ok = (target >= 0) & (target < W.shape[0])
    assert (loss[~ok] == 0).all()
    return loss, lse


def _check_grad(hs, X, W, target, weight, lse, **kw):
    print(f"[loss grad {tuple(X.shape)} x {W.shape[0]}]", flush=True)
    got = hs.token_loss_grad(X, W, target, lse, weight, **kw)
    torch.cuda.synchronize()
    want, size = ref.loss_grad(X, W, target, weight)
    logit = LOGIT * (X.cpu().double().nan_to_num(0, 0, 0).abs() @ W.cpu().double().abs().t()).max().item()
    for name, a, b, s in zip(("dX", "dW"), got, want, size):
        if a is None:
            continue
        bound = ROUND * b.abs() + (ROUND + logit + 2.0 ** -15) * s + RANGE
        assert ((a.cpu().double() - b).abs() <= bound).all(), name
        # the bound on each element is loose where its terms cancel: all together are not
        assert (a.cpu().double() - b).norm() <= 2.0 ** -8 * b.norm() + 1e-300, name
    return got


CASES = [(1, 16, 1), (1, 16, 2), (1, 64, 300), (5, 16, 17), (63, 144, 1000), (64, 64, 128), (130, 272, 4099),
         (257, 64, 259), (300, 1040, 2500), (4100, 32, 4200)]


@pytest.mark.parametrize("T,d,V", CASES)
def test_loss_and_gradient_match_64_bits(hs, T, d, V):
    X, W, target, weight = _problem(T, d, V, seed=T + d + V)
    _, lse = _check_loss(hs, X, W, target)
    _check_grad(hs, X, W, target, weight, lse)


def test_gradient_over_several_pieces_of_the_vocabulary(hs):
    """Enough tokens that one piece of g does not take the vocabulary: three
    pieces, the last one ragged."""
    T, d, V = 65600, 16, 10007
    X, W, target, weight = _problem(T, d, V, seed=4)
    loss, lse = hs.token_loss(X, W, target)
    dX, dW = hs.token_loss_grad(X, W, target, lse, weight)
    torch.cuda.synchronize()
    # in blocks of tokens, on the GPU in float64
    want_dX = torch.empty((T, d), dtype=torch.float64, device=DEV)
    want_dW = torch.zeros((V, d), dtype=torch.float64, device=DEV)
    W64 = W.double()
    Wt = W64.t().contiguous()
    for t in range(0, T, 8200):
        x, y, w = X[t:t + 8200].double(), target[t:t + 8200], weight[t:t + 8200].double()
        ok = (y >= 0) & (y < V)
        logits = x @ Wt
        l64 = torch.logsumexp(logits, -1)
        assert ((lse[t:t + 8200].double() - l64).abs() <= 1e-5).all()
        g = (logits - l64[:, None]).exp()
        k = ok.nonzero()[:, 0]
        g[k, y[k]] -= 1.0
        g *= torch.where(ok, w, 0.0)[:, None]
        want_dX[t:t + 8200] = g @ W64
        want_dW += g.t().contiguous() @ x
    for a, b in ((dX, want_dX), (dW, want_dW)):
        assert (a.double() - b).norm() <= 2.0 ** -8 * b.norm()


def test_large_logits_and_a_single_word(hs):
    """Logits of several hundred, far beyond the range of exp; and a
    vocabulary of one word, whose loss and gradient are 0."""
    X, W, target, weight = _problem(70, 64, 333, seed=5, std=300.0)
    _, lse = _check_loss(hs, X, W, target)
    _check_grad(hs, X, W, target, weight, lse)
    loss, lse = hs.token_loss(X, W[:1], torch.zeros_like(target))
    dX, dW = hs.token_loss_grad(X, W[:1], torch.zeros_like(target), lse, weight)
    torch.cuda.synchronize()
    assert (loss == 0).all() and (dX == 0).all() and (dW == 0).all()


def test_tokens_that_are_not_scored_may_hold_anything(hs):
    X, W, target, weight = _problem(140, 48, 500, seed=6)
    loss, lse = hs.token_loss(X, W, target)
    plain = hs.token_loss_grad(X, W, target, lse, weight)
    off = ~((target >= 0) & (target < 500))
    off[6] = True  # weight 0
    X = X.clone()
    X[off] = float("nan")
    X[off.nonzero()[0]] = float("inf")
    loss2, lse2 = hs.token_loss(X, W, target)
    got = hs.token_loss_grad(X, W, target, lse2, weight)
    torch.cuda.synchronize()
    assert torch.equal(loss2[~off], loss[~off]) and torch.equal(lse2[~off], lse[~off])
    assert (loss2[off & (target < 0)] == 0).all()
    assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])
    assert (got[0][off] == 0).all()


def test_no_scored_token_gives_zeros(hs):
    X, W, target, weight = _problem(40, 32, 90, seed=7)
    target.fill_(-1)
    loss, lse = hs.token_loss(X, W, target)
    dX, dW = hs.token_loss_grad(X, W, target, lse, weight)
    e = X[:0]
    l0, s0 = hs.token_loss(e, W, target[:0])
    dX0, dW0 = hs.token_loss_grad(e, W, target[:0], s0, weight[:0])
    torch.cuda.synchronize()
    assert (loss == 0).all() and (dX == 0).all() and (dW == 0).all() and torch.isfinite(lse).all()
    assert l0.shape == (0,) and dX0.shape == (0, 32) and (dW0 == 0).all()


def test_strided_rows_parts_and_any_workspace(hs):
    T, d, V = 200, 80, 700
    X, W, target, weight = _problem(T, d, V, seed=8)
    loss, lse = _check_loss(hs, X, W, target)
    dX, dW = _check_grad(hs, X, W, target, weight, lse)
    wide = torch.full((T, 120), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 16:96] = X
    out = torch.full((T, 100), 3.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((hs.token_loss_workspace_bytes(T, d, V),), 0xFF, dtype=torch.uint8, device=DEV)
    wg = torch.full((hs.token_loss_grad_workspace_bytes(T, d, V),), 0xFF, dtype=torch.uint8, device=DEV)
    loss2, lse2 = hs.token_loss(wide[:, 16:96], W, target, workspace=ws)
    a, none = hs.token_loss_grad(wide[:, 16:96], W, target, lse, weight, dX=out[:, 8:88], need_dW=False, workspace=wg)
    none2, b = hs.token_loss_grad(X, W, target, lse, weight, need_dX=False, workspace=wg)
    torch.cuda.synchronize()
    assert none is None and none2 is None
    assert torch.equal(loss2, loss) and torch.equal(lse2, lse) and torch.equal(a, dX) and torch.equal(b, dW)
    assert (out[:, :8] == 3.0).all() and (out[:, 88:] == 3.0).all()


def test_gradient_against_differences_of_the_loss(hs):
    """Along a direction D: sum w loss(X + e D) - sum w loss(X - e D) = 2 e <dX, D>
    (and the same for W).  Values lie on a grid of 2^-6 so that the steps of
    e = 2^-6 are exact.  Third-order term: e^2 / 6 of a third derivative of at
    most (2 |D| |W|)^3, here below 2e-3 of the sum; fp32 losses: 2^-20 / e."""
    T, d, V = 64, 64, 600
    g = torch.Generator().manual_seed(12)
    X = (torch.randint(-64, 65, (T, d), generator=g) / 64.0).bfloat16().to(DEV)
    W = (torch.randint(-16, 17, (V, d), generator=g) / 64.0).bfloat16().to(DEV)
    target = torch.randint(0, V, (T,), generator=g).to(DEV)
    weight = (torch.rand(T, generator=g) / T).to(DEV)
    e = 2.0 ** -6
    _, lse = hs.token_loss(X, W, target)
    dX, dW = hs.token_loss_grad(X, W, target, lse, weight)

    def total(X, W):
        return (hs.token_loss(X, W, target)[0].double() * weight.double()).sum().item()

    for of, grad in (("X", dX), ("W", dW)):
        D = torch.sign(grad.double())  # the direction of steepest ascent in steps of e
        step = (e * D).bfloat16()
        if of == "X":
            diff = total(X + step, W) - total(X - step, W)
        else:
            diff = total(X, W + step) - total(X, W - step)
        along = (grad.double() * D).sum().item()
        assert math.isclose(diff / (2 * e), along, rel_tol=1e-2), (of, diff / (2 * e), along)


def test_loss_and_gradient_replay_in_a_graph(hs):
    T, d, V = 300, 64, 900
    X, W, target, weight = _problem(T, d, V, seed=9)
    loss, lse = hs.token_loss(X, W, target)
    want = [loss.clone(), lse.clone(), *(t.clone() for t in hs.token_loss_grad(X, W, target, lse, weight))]
    out = [torch.empty_like(t) for t in want]
    ws = torch.empty(max(hs.token_loss_workspace_bytes(T, d, V), hs.token_loss_grad_workspace_bytes(T, d, V)),
                     dtype=torch.uint8, device=DEV)

    def call():
        hs.token_loss(X, W, target, loss=out[0], lse=out[1], workspace=ws)
        hs.token_loss_grad(X, W, target, out[1], weight, dX=out[2], dW=out[3], workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        for t in out:
            t.zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), f"replay {i}"
