"""The tiles and splits that the other tests' sizes do not take, with enough k
in each for its ring of stages to turn, against 64 bits on the GPU.  That all of
them together take every way is checked in test_adapt_routes_covered.py."""
from __future__ import annotations

import pytest
import torch

from tests.test_gpu_adapt import S_G, _bf, _gen, _low, _problem
from tests.test_gpu_loss import LOGIT
from tests.test_gpu_loss_precision import _exact, _problem as _loss_problem

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"

LINEAR = [  # tokens, in, out, adapters, rank
    (9, 192, 26, 16, 32), (20, 1824, 161, 9, 64), (23, 288, 38, 6, 24), (28, 80, 84, 32, 24), (42, 4352, 58, 36, 8),
    (44, 224, 45, 4, 232), (48, 7344, 23, 50, 112), (58, 2912, 120, 11, 16), (59, 160, 75, 13, 16),
    (712, 10048, 29, 3, 224), (662, 160, 648, 2, 48), (270, 2688, 47, 2, 8), (202, 192, 35, 3, 40),
    (2316, 2096, 44, 2, 72), (1200, 4096, 512, 4, 16), (5414, 3584, 144, 52, 48), (4727, 9184, 947, 2, 136),
    (1040, 14336, 4096, 8, 32), (2316, 2096, 44, 0, 0), (5414, 3584, 144, 0, 0), (4083, 640, 1069, 0, 0),
    (4727, 9184, 947, 0, 0), (4524, 288, 6968, 0, 0), (8192, 1040, 2064, 4, 16)]
GRAD = [  # tokens, in, out, adapters, rank
    (1, 10928, 1087, 6, 24), (1508, 2992, 136, 17, 8), (2047, 4096, 4096, 1, 16), (132, 11040, 3781, 5, 16),
    (4100, 2064, 1040, 4, 64)]
LOSS = [  # tokens, d, vocabulary
    (11, 2640, 7257), (14, 3616, 4201), (372, 1024, 6921), (17, 5568, 17224), (805, 8080, 72), (135, 2672, 11489),
    (6745, 4992, 78), (497, 80, 15849), (1026, 160, 3728), (200, 2064, 33000), (2050, 2064, 4099),
    (40, 2064, 2000), (2048, 4096, 32000), (64, 1024, 128000), (384, 1024, 8192)]


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def _weights(codes, packed):
    """float64 [out, in] of the stored layer, on the GPU."""
    codes = codes.long()
    e, f = codes >> 3, (codes & 7).double()
    S = torch.where(e == 0, f * 2.0 ** -9, (8 + f) * torch.exp2(e.double() - 10.0)) * float(torch.tensor(S_G))
    nibbles = torch.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[0], -1).long()
    v = torch.cat([GRID, -GRID]).to(DEV)[nibbles]
    return v * S.repeat_interleave(16, 1)


def _layer64(X, W, low):
    """(Y, the sums of the absolute terms behind it)."""
    Y, size = X @ W.t().contiguous(), X.abs() @ W.abs().t().contiguous()
    if low["A"] is not None:
        A, B = low["A"].double(), low["B"].double()
        for a in range(A.shape[0]):
            t = (low["adapter"] == a).nonzero()[:, 0]
            s, down, up = low["alpha"][a].double(), A[a].t().contiguous(), B[a].t().contiguous()
            Y[t] += s * (X[t] @ down) @ up
            size[t] += s.abs() * (X[t].abs() @ down.abs()) @ up.abs()
    return Y, size


def _grad64(dY, X, W, low):
    A, B = low["A"].double(), low["B"].double()
    out = []
    for f in (lambda t: t, torch.abs):
        d, x, w = f(dY), f(X), f(W)
        dX, dA, dB = d @ w, torch.zeros_like(A), torch.zeros_like(B)
        for a in range(A.shape[0]):
            t = (low["adapter"] == a).nonzero()[:, 0]
            s, u, v = f(low["alpha"][a].double()), f(A[a]), f(B[a])
            down = s * d[t] @ v
            dX[t] += down @ u
            dA[a] = down.t().contiguous() @ x[t]
            dB[a] = d[t].t().contiguous() @ (s * x[t] @ u.t().contiguous())
        out.append((dX, dA, dB))
    return out


def _close(got, want, size, k, what):
    """One rounding to bf16, at most 2^-8 of the value.  Before it fp32 sums of
    chains of k / 16 products and up to 32 splits, each 2^-24 of the sum of
    absolute terms, and 2^-16 of it where u and v enter in two bf16 parts."""
    bound = 2.0 ** -8 * want.abs() + ((k / 16 + 32) * 2.0 ** -24 + 2.0 ** -16) * size
    assert got.shape == want.shape and ((got.double() - want).abs() <= bound).all(), what


@pytest.mark.parametrize("T,n,m,count,rank", LINEAR)
def test_layer(hs, T, n, m, count, rank):
    p = _problem(T, n, m, count, rank, seed=T + n + m, how="runs" if T > 1000 else "each")
    print(f"[linear {T} x {n} -> {m}, {count} adapters of rank {rank}]", flush=True)
    got = hs.adapted_linear(p["X"], S_G, p["codes"], p["packed"], **_low(p))
    torch.cuda.synchronize()
    want, size = _layer64(p["X"].double(), _weights(p["codes"], p["packed"]), _low(p))
    _close(got, want, size, n + 2 * rank, "Y")


@pytest.mark.parametrize("T,n,m,count,rank", GRAD)
def test_gradients(hs, T, n, m, count, rank):
    p = _problem(T, n, m, count, rank, seed=T + n + m, how="runs" if T > 1000 else "each")
    dY = _bf((T, m), 1.0, _gen(T))
    q, scale = hs.pack_activations(p["X"])
    X = hs.unpack_activations(q, scale).double()
    print(f"[grad {T} x {n} -> {m}, {count} adapters of rank {rank}]", flush=True)
    got = hs.adapted_linear_grad(dY, q, scale, S_G, p["codes"], p["packed"], **_low(p))
    torch.cuda.synchronize()
    want, size = _grad64(dY.double(), X, _weights(p["codes"], p["packed"]), _low(p))
    for name, a, b, s, k in zip(("dX", "dA", "dB"), got, want, size, (m + 2 * rank, T + m, T + n)):
        _close(a, b, s, k, name)


@pytest.mark.parametrize("T,d,V", LOSS)
def test_loss_and_its_gradient(hs, T, d, V):
    """The gradient's bounds are those of test_gpu_loss_precision.py."""
    X, W, target, weight = _loss_problem(T, d, V, 0.1, seed=T + V)
    target[T // 2] = V - 1
    print(f"[loss {T} x {d} over {V}]", flush=True)
    loss, lse = hs.token_loss(X, W, target)
    got = hs.token_loss_grad(X, W, target, lse, weight)
    torch.cuda.synchronize()
    logits = X.double() @ W.double().t().contiguous()
    want_lse = torch.logsumexp(logits, -1)
    scored = target >= 0
    want = torch.where(scored, want_lse - logits.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    size = (X.double().abs() @ W.double().abs().t().contiguous()).amax(-1)
    tol = 2 * LOGIT * size + 2.0 ** -20 * (1.0 + logits.abs().amax(-1)) + 2.0 ** -20  # as test_gpu_loss.py
    assert ((lse.double() - want_lse).abs() <= tol).all() and ((loss.double() - want).abs() <= tol).all()
    del logits, size
    exact, spread, _, largest = _exact(X, W, target, weight)
    for name, a, b, s in zip(("dX", "dW"), got, exact, spread):
        error = ((a.double() - b).norm() / b.norm()).item()
        apart = ((a.double() - b.bfloat16().double()).norm() / b.norm()).item()
        off = (d / 16 + 2) ** 0.5 * 2.0 ** -24 * largest * (s.norm() / b.norm()).item()
        delta = 2.0 ** -16 + off
        assert error <= 2.0 ** -8 / 3 ** 0.5 * 1.02 + off, (name, error)
        assert apart <= (2.0 * delta * 2.0 ** -7) ** 0.5 + delta, (name, apart)
