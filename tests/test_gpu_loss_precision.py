"""How exact the token loss's gradient is where the softmax is peaked, as in
training, against 64 bits."""
from __future__ import annotations

import pytest
import torch

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


def _problem(T, d, V, pull, seed):
    """Hidden states that lean towards their target's row of W by `pull`: from a
    softmax spread over all words (0) to one that is nearly sure."""
    g = torch.Generator().manual_seed(seed)
    W = torch.randn((V, d), generator=g) * 2.0 * d ** -0.5
    target = torch.randint(0, V, (T,), generator=g)
    X = torch.randn((T, d), generator=g) + pull * W[target] * d ** 0.5 / 2.0
    target[torch.rand(T, generator=g) < 0.125] = -100
    weight = (target >= 0).float() / (target >= 0).sum()
    return X.bfloat16().to(DEV), W.bfloat16().to(DEV), target.to(DEV), weight.to(DEV)


def _exact(X, W, target, weight):
    X, W = X.double(), W.double()
    scored = target >= 0
    g = torch.softmax(X @ W.t().contiguous(), -1)
    k = scored.nonzero()[:, 0]
    loss = -g[k, target[k]].log().mean().item()
    w = torch.where(scored, weight.double(), 0.0)[:, None]
    spread = (g * w) @ W.abs(), (g * w).t().contiguous() @ X.abs()
    g[k, target[k]] -= 1.0
    g *= w
    return (g @ W, g.t().contiguous() @ X), spread, loss, (X @ W.t().contiguous()).abs().max().item()


# Few tokens whose k is split; 128, 256 and more tokens; several tile sizes.
@pytest.mark.parametrize("pull", [0.0, 0.15, 0.3, 0.5, 0.8])
@pytest.mark.parametrize("T,d,V", [(64, 512, 4000), (65, 512, 4000), (130, 512, 300), (512, 512, 4000), (2050, 256, 9001)])
def test_gradients_are_rounded_to_bf16_once(hs, T, d, V, pull):
    """One rounding to bf16 errs by at most 2^-8 / sqrt(3) of the norm (uniform
    in a unit of 2^-7 of a value's power of two).  Before it a value is off by at
    most 2^-16 of itself (two bf16 parts, 2^-17, and fp32 sums) and by what the
    logits in fp32 leave: d / 16 roundings of a sum, one of lse and one of their
    difference, each of 2^-24 of the largest logit and in no common direction,
    which change p by as much of itself (near a softmax of 1 that is more than
    1 - p).  Of values rounded from 64 bits only those differ that lie as near
    (delta) to a boundary, a share of 2 delta over the unit, each by the unit:
    together sqrt(2 delta 2^-7) of the norm."""
    X, W, target, weight = _problem(T, d, V, pull, seed=T + V)
    _, lse = hs.token_loss(X, W, target)
    got = hs.token_loss_grad(X, W, target, lse, weight)
    torch.cuda.synchronize()
    exact, spread, mean, largest = _exact(X, W, target, weight)
    for name, a, b, s in zip(("dX", "dW"), got, exact, spread):
        error = ((a.double() - b).norm() / b.norm()).item()
        apart = ((a.double() - b.bfloat16().double()).norm() / b.norm()).item()
        logits = (d / 16 + 2) ** 0.5 * 2.0 ** -24 * largest * (s.norm() / b.norm()).item()
        print(f"{name} at a mean loss of {mean:.2f}: {error:.5f} of the norm, {apart:.6f} from rounded; "
              f"logits {logits:.6f}", flush=True)
        delta = 2.0 ** -16 + logits
        assert error <= 2.0 ** -8 / 3 ** 0.5 * 1.02 + logits, name
        assert apart <= (2.0 * delta * 2.0 ** -7) ** 0.5 + delta, name
