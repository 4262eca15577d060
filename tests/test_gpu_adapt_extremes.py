"""Checkpoints whose blocks reach the ends of bf16's range, and gradients at
them, against 64-bit plain implementations."""
from __future__ import annotations

import pytest
import torch

from tests import adapt_ref as ref
from tests.test_gpu_adapt import _bf, _check_grad, _gen, _low, _problem

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"
LARGEST = torch.tensor([0x7F7F, 0x7F7E, 0x7F7D, 0x7F00], dtype=torch.int16).view(torch.bfloat16)


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


@pytest.mark.parametrize("n", [16, 144, 1040])
def test_blocks_with_the_largest_finite_values_are_restored(hs, n):
    """bf16(fp32(q scale)) bit for bit: the largest magnitudes of both signs,
    each alone in its block or beside zeros, halves and tiny values."""
    X = torch.zeros((4 * len(LARGEST), n), dtype=torch.bfloat16)
    for k, top in enumerate(LARGEST):
        for row, (sign, rest) in enumerate(((1, 0.0), (-1, 0.0), (1, 0.5), (-1, -2.0 ** -100))):
            X[4 * k + row] = (top.float() * rest).bfloat16()
            X[4 * k + row, 3::128] = sign * top
    X = X.to(DEV)
    q, scale, back = ref.pack(X)
    assert torch.isfinite(back.float()).all()
    got_q, got_scale = hs.pack_activations(X)
    got = hs.unpack_activations(got_q, got_scale)
    torch.cuda.synchronize()
    assert torch.equal(got_q.cpu(), q) and torch.equal(got_scale.cpu(), scale) and torch.equal(got.cpu(), back)


@pytest.mark.parametrize("T,rank", [(70, 16), (70, 64), (600, 16), (600, 64)])
def test_gradients_at_a_checkpoint_with_the_largest_finite_values(hs, T, rank):
    """One token in ten has such blocks.  A and dY are scaled so that u, dA and
    dB stay within range."""
    n, m = 272, 48
    p = _problem(T, n, m, 2, rank, seed=T + rank)
    p["X"][::10] = 0.0
    p["X"][::10, 5] = LARGEST[0].to(DEV)
    p["X"][5::10, 200] = -LARGEST[1].to(DEV)
    p["A"] *= 2.0 ** -60
    p["adapter"][::10] = 1
    dY = _bf((T, m), 2.0 ** -60, _gen(T))
    _, dA, dB = _check_grad(hs, p, dY)
    assert torch.isfinite(dA.float()).all() and torch.isfinite(dB.float()).all()
