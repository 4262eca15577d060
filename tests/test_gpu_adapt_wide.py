"""Few tokens with adapters of large rank over many outputs, whose adapters' part
goes through the product's own stages, against 64 bits on the GPU."""
from __future__ import annotations

import pytest
import torch

from tests.test_gpu_adapt import S_G, _low, _problem
from tests.test_gpu_adapt_tiles import _close, _layer64, _weights

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

LINEAR = [  # tokens, in, out, adapters, rank
    (16, 160, 21000, 3, 256), (16, 144, 21000, 2, 256), (16, 5056, 21000, 2, 256), (16, 3728, 21000, 2, 256),
    (30, 160, 13437, 3, 256), (30, 144, 13437, 2, 256), (30, 5056, 13437, 2, 232), (30, 3728, 13437, 2, 256),
    (45, 160, 13437, 23, 224), (45, 528, 10312, 3, 192), (45, 4320, 15073, 6, 224), (45, 3728, 14353, 28, 176),
    (61, 160, 13437, 2, 256), (61, 144, 13437, 40, 136), (61, 11104, 12554, 1, 144), (61, 2064, 13000, 4, 256)]


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    return hs


@pytest.mark.parametrize("T,n,m,count,rank", LINEAR)
def test_layer(hs, T, n, m, count, rank):
    p = _problem(T, n, m, count, rank, seed=T + n + m)
    print(f"[linear {T} x {n} -> {m}, {count} adapters of rank {rank}]", flush=True)
    got = hs.adapted_linear(p["X"], S_G, p["codes"], p["packed"], **_low(p))
    torch.cuda.synchronize()
    want, size = _layer64(p["X"].double(), _weights(p["codes"], p["packed"]), _low(p))
    _close(got, want, size, n + 2 * rank, "Y")
