"""Calls of a layer of stored experts that go in several pieces: a token's bits
are those of its call, whichever piece it lies in."""
from __future__ import annotations

import pytest
import torch

from tests.test_gpu_experts import DEV, _gen, _problem, hs  # noqa: F401

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

# One wave to a row and several; more tokens than a piece of 4096 / k takes, the
# last piece short enough that alone it would take another tile, other waves a
# row or other splits of the down product.
CALLS = [(2100, 2048, 2048, 8, 2), (683, 2048, 1024, 64, 6), (686, 1040, 1024, 5, 6), (4097, 528, 1296, 3, 1),
         (2051, 1296, 528, 2, 2), (130, 528, 1040, 9, 32), (2100, 2048, 128, 5, 2), (2100, 528, 64, 500, 2)]


@pytest.mark.parametrize("T,n,hidden,E,k", CALLS)
def test_a_token_has_the_same_bits_in_every_piece(hs, T, n, hidden, E, k):  # noqa: F811
    p = _problem(T, n, hidden, E, k, ids="distinct" if k <= E else "wild")
    print(f"[pieces {T} {n} {hidden} {E} {k}]", flush=True)
    whole = hs.expert_layer(**p)
    for by in (1, T // 2, T - 4096 // k):  # the last piece's tokens come from another one
        order = torch.arange(T, device=DEV).roll(by)
        mixed = dict(p, X=p["X"][order], expert=p["expert"][order], weight=p["weight"][order])
        assert torch.equal(hs.expert_layer(**mixed), whole[order]), by


@pytest.mark.parametrize("ld", [1 << 19, 1 << 21])
def test_rows_far_apart_change_no_bits(hs, ld):  # noqa: F811
    """X is addressed in 32 bits: rows far apart make the pieces smaller."""
    T, n, hidden, E, k = 1029, 1040, 1024, 6, 2
    p = _problem(T, n, hidden, E, k)
    whole = hs.expert_layer(**p)
    X = torch.zeros((T - 1) * ld + n, dtype=torch.bfloat16, device=DEV).as_strided((T, n), (ld, 1))
    X.copy_(p["X"])
    assert torch.equal(hs.expert_layer(**dict(p, X=X)), whole)


@pytest.mark.parametrize("T,n,hidden,E,k", [(1, 528, 1040, 8, 2), (90, 528, 1040, 8, 2)] + CALLS[1:])
def test_a_workspace_of_the_size_asked_for_is_enough(hs, T, n, hidden, E, k):  # noqa: F811
    """What lies behind it is left as it was."""
    p = _problem(T, n, hidden, E, k, ids="distinct" if k <= E else "wild")
    need = hs.expert_layer_workspace_bytes(T, n, hidden, E, k)
    buf = torch.randint(0, 256, (need + 65536,), generator=_gen(T), dtype=torch.int32).to(torch.uint8).to(DEV)
    behind = buf[need:].clone()
    got = hs.expert_layer(**p, workspace=buf[:need])
    assert torch.equal(got, hs.expert_layer(**p))
    assert torch.equal(buf[need:], behind)
