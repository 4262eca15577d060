"""Calls given another stream than the current one, with memory of their own:
work that is still queued on either stream neither writes to it nor is written
over by it."""
from __future__ import annotations

import pytest
import torch

from tests.test_gpu_adapt import S_G, _bf, _gen, _low, _problem
from tests.test_gpu_loss import _problem as _loss_problem

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"
WAIT = 50_000_000  # cycles of a spin that keeps a stream busy, some ten milliseconds


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


def _calls(hs):
    T, n, m, count, rank, V = 700, 1040, 300, 3, 24, 900
    p = _problem(T, n, m, count, rank, seed=31)
    layer = S_G, p["codes"], p["packed"]
    dY = _bf((T, m), 1.0, _gen(3))
    q, scale = hs.pack_activations(p["X"])
    X, W, target, weight = _loss_problem(T, 64, V, seed=3)
    _, lse = hs.token_loss(X, W, target)
    h = hs.hdiag(p["X"])
    dense = _bf((m, n), 0.02, _gen(4))
    return {
        "adapted_linear": lambda s: [hs.adapted_linear(p["X"], *layer, **_low(p), stream=s)],
        "pack_activations": lambda s: list(hs.pack_activations(p["X"], stream=s)),
        "unpack_activations": lambda s: [hs.unpack_activations(q, scale, stream=s)],
        "adapted_linear_grad": lambda s: list(hs.adapted_linear_grad(dY, q, scale, *layer, **_low(p), stream=s)),
        "token_loss": lambda s: list(hs.token_loss(X, W, target, stream=s)),
        "token_loss_grad": lambda s: list(hs.token_loss_grad(X, W, target, lse, weight, stream=s)),
        "hdiag": lambda s: [hs.hdiag(p["X"], stream=s)],
        "search": lambda s: list(hs.search(dense, h, S_G, down=2, up=2, stream=s)),
        "output_error": lambda s: [hs.output_error(p["X"], dense, *layer, stream=s)],
    }


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("fn", ["adapted_linear", "pack_activations", "unpack_activations", "adapted_linear_grad",
                                "token_loss", "token_loss_grad", "hdiag", "search", "output_error"])
def test_a_call_on_a_busy_side_stream_keeps_its_memory(hs, fn, handle):
    """The call waits on its stream while the current stream allocates and
    fills as much memory as it frees; then the other way round."""
    call = _calls(hs)[fn]
    want = [t.clone() for t in call(None)]
    side = torch.cuda.Stream()
    stream = side.cuda_stream if handle else side
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(WAIT)
    got = call(stream)
    junk = [torch.full((k << 20,), 0x5A, dtype=torch.uint8, device=DEV) for k in (1, 1, 1, 2, 2, 4, 8, 16, 32)]
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all((t == 0x5A).all() for t in junk)
    del junk, got
    torch.cuda._sleep(WAIT)  # what the current stream queues from here on comes later
    got = call(stream)
    side.synchronize()
    copies = []
    with torch.cuda.stream(side):
        copies = [t.clone() for t in got]
    side.synchronize()
    assert all(torch.equal(a.cpu(), b.cpu()) for a, b in zip(copies, want))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
