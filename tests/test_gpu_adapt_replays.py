"""Captured calls read their inputs at the replay: activations, each token's
adapter, targets and weights are written anew between replays, and every replay
gives the bits of an eager call on what is there."""
from __future__ import annotations

import pytest
import torch

from tests.test_gpu_adapt import DEV, S_G, _bf, _gen, _ids, _low, _problem
from tests.test_gpu_loss import _problem as _loss_problem

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


def _replays(call, out, write, count=5):
    """call(out) is captured; write(i) puts new inputs in place before replay i."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    before = None
    for i in range(count):
        write(i)
        want = [torch.empty_like(t) for t in out]
        call(want)
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), f"replay {i}"
        assert before is None or any(not torch.equal(a, b) for a, b in zip(want, before)), f"replay {i} repeats"
        before = want


def _new_adapters(p, T, count, i):
    """Another set each time: every token its own, none at all, one for all, runs."""
    p["adapter"].copy_(_ids(T, count, _gen(50 + i), ("each", "none", "each", "runs", "each")[i]))
    if i == 2:
        p["adapter"].fill_(count - 1)
    p["alpha"].copy_(torch.randn(count, generator=_gen(60 + i)))


@pytest.mark.parametrize("T,n,m", [(1, 1040, 300), (48, 528, 700), (300, 2064, 130), (700, 1040, 300), (1100, 272, 520)])
def test_layer(hs, T, n, m):
    count = 5
    p = _problem(T, n, m, count, 24, seed=T)
    ws = torch.empty(hs.adapted_linear_workspace_bytes(T, n, m, count, 24), dtype=torch.uint8, device=DEV)

    def write(i):
        p["X"].copy_(_bf((T, n), 1.0 + i, _gen(70 + i)))
        _new_adapters(p, T, count, i)
        ws.fill_(0xFF)

    _replays(lambda o: hs.adapted_linear(p["X"], S_G, p["codes"], p["packed"], **_low(p), Y=o[0], workspace=ws),
             [torch.empty((T, m), dtype=torch.bfloat16, device=DEV)], write)


@pytest.mark.parametrize("T,n,m", [(40, 272, 100), (300, 144, 96), (1500, 528, 272)])
def test_checkpoint_and_gradients(hs, T, n, m):
    count, rank = 4, 16
    p = _problem(T, n, m, count, rank, seed=T)
    dY = _bf((T, m), 1.0, _gen(8))
    q, scale = hs.pack_activations(p["X"])
    ws = torch.empty(hs.adapted_linear_grad_workspace_bytes(T, n, m, count, rank), dtype=torch.uint8, device=DEV)

    def write(i):
        p["X"].copy_(_bf((T, n), 1.0 + i, _gen(70 + i)))
        dY.copy_(_bf((T, m), 2.0 ** -i, _gen(80 + i)))
        _new_adapters(p, T, count, i)
        ws.fill_(0xFF)

    def call(o):
        hs.pack_activations(p["X"], q=q, scale=scale)
        hs.adapted_linear_grad(dY, q, scale, S_G, p["codes"], p["packed"], **_low(p), dX=o[0], dA=o[1], dB=o[2],
                               workspace=ws)

    _replays(call, [torch.empty((T, n), dtype=torch.bfloat16, device=DEV), torch.empty_like(p["A"]),
                    torch.empty_like(p["B"])], write)


@pytest.mark.parametrize("T,d,V", [(20, 2048, 300), (60, 64, 900), (300, 64, 900), (700, 272, 4099)])
def test_loss_and_gradient(hs, T, d, V):
    X, W, target, weight = _loss_problem(T, d, V, seed=9)
    ws = torch.empty(max(hs.token_loss_workspace_bytes(T, d, V), hs.token_loss_grad_workspace_bytes(T, d, V)),
                     dtype=torch.uint8, device=DEV)

    def write(i):
        new = _loss_problem(T, d, V, seed=90 + i, std=1.0 + i)
        for old, t in zip((X, target, weight), (new[0], new[2], new[3])):
            old.copy_(t)
        weight.mul_(4.0 ** (i - 2))  # another largest weight
        if i == 3:
            target.fill_(-100)
        ws.fill_(0xFF)

    def call(o):
        hs.token_loss(X, W, target, loss=o[0], lse=o[1], workspace=ws)
        hs.token_loss_grad(X, W, target, o[1], weight, dX=o[2], dW=o[3], workspace=ws)

    _replays(call, [torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty_like(X), torch.empty_like(W)],
             write)
