"""A stored layer without adapters for few tokens: rows that one pass writes,
and rows whose k is split, against 64 bits."""
from __future__ import annotations

import pytest
import torch

from tests.test_gpu_adapt import S_G, _check_linear, _problem

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


@pytest.mark.parametrize("T", [1, 16, 17, 40, 64, 65])
@pytest.mark.parametrize("n,m", [(16, 1), (512, 515), (48, 2050), (4096, 130), (4112, 1027)])
def test_matches_64_bits_in_rows_of_any_stride(hs, T, n, m):
    p = _problem(T, n, m, 0, 0, seed=T + n + m)
    plain = _check_linear(hs, p)
    for lead, ld in ((0, m + 3), (4, m + 8), (1, m + 1)):
        out = torch.full((T, ld + lead), 7.0, dtype=torch.bfloat16, device=DEV)
        hs.adapted_linear(p["X"], S_G, p["codes"], p["packed"], Y=out[:, lead:lead + m])
        torch.cuda.synchronize()
        assert torch.equal(out[:, lead:lead + m], plain)
        assert (out[:, :lead] == 7.0).all() and (out[:, lead + m:] == 7.0).all()


@pytest.mark.parametrize("T,n,m", [(1, 512, 64), (48, 512, 300), (20, 4096, 100)])
def test_tokens_without_an_adapter_are_the_layer_alone(hs, T, n, m):
    """The same values as with adapters that no token uses, up to the order of
    the sums."""
    p = _problem(T, n, m, 2, 8, seed=9, how="none")
    with_none = _check_linear(hs, p)
    p.update(A=None, B=None, alpha=None, adapter=None)
    alone = _check_linear(hs, p)
    assert (alone.float() - with_none.float()).norm() <= 2.0 ** -8 * with_none.float().norm()
