"""What the library's plans of the stored layer in use ask of a caller (CPU
only; sizes alone)."""
import subprocess
from pathlib import Path

import pytest

from paper_2608_28113_amd import _lib, build

ROOT = Path(__file__).resolve().parent.parent


@pytest.fixture(scope="module")
def L():
    if not _lib.LIB_PATH.exists():
        build.build()
    _lib.load()
    return _lib


@pytest.mark.parametrize("T", [1, 16, 33, 64, 65, 512])
def test_few_tokens_without_adapters_write_their_result_in_one_pass(L, T):
    """Nothing is split in a row of up to 512 and no adapter's part is added:
    there is nothing to keep in between."""
    assert all(L.hscale_adapted_linear_workspace_bytes(T, n, m, 0, 0) == 0 for n in (16, 512) for m in (1, 24, 14336))


A = 1 << 44  # fake but aligned device addresses, far apart
OVERLAP, WORKSPACE = -8, -6


def _linear(L, t, n, m, count, rank, ws):
    """Y lies on X: refused for that once the workspace is large enough."""
    ad = (count, rank, 10 * A, 11 * A, 12 * A, 13 * A) if count else None
    return L.hscale_adapted_linear(A, t, n, n, m, 1e-3, 2 * A, 3 * A, ad, A, m, 5 * A, ws, 0)


def _grad(L, t, n, m, count, rank, ws):
    """Rows of dY that are not whole 16-byte words take the most."""
    ad = (count, rank, 10 * A, 11 * A, 12 * A, 13 * A)
    return L.hscale_adapted_linear_grad(A, t, m, m + 1, 2 * A, 3 * A, n, 1e-3, 4 * A, 5 * A, ad, A, n, 7 * A, 8 * A, 9 * A,
                                        ws, 0)


def _loss(L, t, d, vocab, count, rank, ws):
    return L.hscale_token_loss(A, t, d, d, 2 * A, vocab, 3 * A, 4 * A, 4 * A, 6 * A, ws, 0)


def _loss_grad(L, t, d, vocab, count, rank, ws):
    return L.hscale_token_loss_grad(A, t, d, d, 2 * A, vocab, 3 * A, 5 * A, 7 * A, A, d, 9 * A, 6 * A, ws, 0)


CALLS = {"adapted_linear": _linear, "adapted_linear_grad": _grad, "token_loss": _loss, "token_loss_grad": _loss_grad}


@pytest.mark.parametrize("fn,T,a,b,count,rank", [
    ("adapted_linear", 512, 4096, 14336, 32, 16), ("adapted_linear", 8192, 14336, 4096, 8, 32),
    ("adapted_linear", 1024, 4096, 4096, 0, 0), ("adapted_linear", 4200, 4096, 1024, 4, 256),
    ("adapted_linear_grad", 8192, 14336, 4096, 4, 64), ("adapted_linear_grad", 2048, 4096, 4096, 1, 16),
    ("token_loss", 512, 1024, 8192, 0, 0), ("token_loss", 4096, 4096, 32003, 0, 0),
    ("token_loss_grad", 8192, 4096, 128000, 0, 0), ("token_loss_grad", 700, 1024, 8192, 0, 0)])
def test_a_workspace_for_many_tokens_serves_every_call_with_fewer(L, fn, T, a, b, count, rank):
    sizes = getattr(L, f"hscale_{fn}_workspace_bytes")
    extra = (count, rank) if fn.startswith("adapted") else ()
    need = sizes(T, a, b, *extra)
    tokens = sorted({*range(1, min(T, 1100) + 1), *range(1, T + 1, 13), T})
    asked = [sizes(t, a, b, *extra) for t in tokens]
    assert asked == sorted(asked) and asked[-1] == need
    assert [CALLS[fn](L, t, a, b, count, rank, need) for t in tokens] == [OVERLAP] * len(tokens)
    if need:
        assert CALLS[fn](L, T, a, b, count, rank, need - 1) == WORKSPACE


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    """The plans alone, built from plan.h."""
    exe = tmp_path_factory.mktemp("plan") / "driver"
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                        str(ROOT / "paper_2608_28113_amd" / "csrc"), "-o", str(exe),
                        str(ROOT / "tests" / "native" / "adapt_plan_driver.cpp")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return exe


def test_no_plan_uses_more_than_its_call_asks_for(driver):
    r = subprocess.run([str(driver)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "plans: ok" in r.stdout, r.stdout + r.stderr
