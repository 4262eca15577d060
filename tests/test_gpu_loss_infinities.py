"""Words whose logits are -inf (a vocabulary with words masked out) in the token
loss, against 64 bits over the other words."""
from __future__ import annotations

import pytest
import torch

from tests import adapt_ref as ref
from tests.test_gpu_loss import LOGIT

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"
MASKS = {
    "the first words": lambda v, V: v < V // 2,
    "the last words": lambda v, V: v >= V // 3,
    "all but the last": lambda v, V: v < V - 1,
    "all but one in the middle": lambda v, V: v != V // 2,
    "runs of four, and of 256": lambda v, V: (v // 4 % 2 == 0) | (v // 256 % 2 == 1),
}


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


# Tiles of each size, and few tokens and words whose logits go through memory.
@pytest.mark.parametrize("mask", sorted(MASKS))
@pytest.mark.parametrize("T,d,V", [(3, 16, 40), (70, 64, 700), (300, 80, 5000), (40, 16, 33000), (2050, 64, 9001), (20, 4096, 500)])
def test_words_of_minus_infinity_count_for_nothing(hs, T, d, V, mask):
    g = torch.Generator().manual_seed(T + V)
    X = torch.randn((T, d), generator=g).bfloat16()
    W = (torch.randn((V, d), generator=g) * 2.0 * d ** -0.5).bfloat16()
    X[:, 0] = 1.0
    off = MASKS[mask](torch.arange(V), V)
    words = (~off).nonzero()[:, 0]
    target = words[torch.randint(0, len(words), (T,), generator=g)]
    target[0] = off.nonzero()[0, 0]  # a masked word: an infinite loss
    masked = W.clone()
    masked[off, 0] = float("-inf")
    print(f"[loss {T} x {d} over {V}, {mask} masked]", flush=True)
    loss, lse = hs.token_loss(X.to(DEV), masked.to(DEV), target.to(DEV))
    torch.cuda.synchronize()
    place = torch.zeros(V, dtype=torch.int64)
    place[words] = torch.arange(len(words))
    want, want_lse, logits = ref.loss(X, W[words], place[target])
    size = (X.double().abs() @ W[words].double().abs().t()).amax(-1)
    tol = 2 * LOGIT * size + 2.0 ** -20 * (1.0 + logits.abs().amax(-1)) + 2.0 ** -20  # as tests/test_gpu_loss.py
    assert ((lse.cpu().double() - want_lse).abs() <= tol).all()
    assert ((loss.cpu().double() - want).abs() <= tol)[1:].all()
    assert loss[0].item() == float("inf")


@pytest.mark.parametrize("T,d,V", [(5, 16, 300), (300, 64, 700), (4, 4096, 300)])
def test_a_word_of_nan_reaches_every_token_and_no_other_value_is_lost(hs, T, d, V):
    g = torch.Generator().manual_seed(V)
    X = torch.randn((T, d), generator=g).bfloat16().to(DEV)
    W = (torch.randn((V, d), generator=g) * d ** -0.5).bfloat16().to(DEV)
    X[:, 0] = 1.0
    W[: V // 2, 0] = float("-inf")
    W[V // 4] = float("nan")
    loss, lse = hs.token_loss(X, W, torch.full((T,), V - 1, device=DEV))
    torch.cuda.synchronize()
    assert loss.isnan().all() and lse.isnan().all()
