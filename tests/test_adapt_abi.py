"""Refusals of the adapted layer, the checkpoints and the token loss: at the C
ABI (fake addresses; nothing here reaches the HIP runtime) and in the torch
front end (`meta` tensors stand in for device tensors, and the library's entry
points for stubs that must not be reached by a bad buffer)."""
import re
import subprocess
from pathlib import Path

import pytest
import torch

from paper_2608_28113_amd import _lib, build, ops
from tests.test_front_end import (SCRATCH, Reached, bf, f32, fake_gpu, flat, i8, on_host,  # noqa: F401
                                  one_more_row, strided, u8, wrong_dtype)

ROOT = Path(__file__).resolve().parent.parent
A = 1 << 30  # fake but aligned device addresses, far apart


@pytest.fixture(scope="module")
def L():
    if not _lib.LIB_PATH.exists():
        build.build()
    _lib.load()
    return _lib


T, n, m, count, rank = 100, 64, 24, 3, 8
AD = (count, rank, 10 * A, 11 * A, 12 * A, 13 * A)


def test_workspace_sizes(L):
    f = L.hscale_adapted_linear_workspace_bytes
    assert f(0, n, m, count, rank) == f(T, 0, m, count, rank) == f(T, n, 0, count, rank) == 0
    assert f(T, 17, m, count, rank) == f(-1, n, m, count, rank) == f(T, n, m, 4097, rank) == 0
    assert f(T, n, m, count, 4) == f(T, n, m, count, 264) == f(T, n, m, -1, rank) == 0
    assert f(T, n, m, 0, 0) == 0  # few tokens of a short row: nothing is split, no adapter
    assert 0 < f(T, n, m, count, rank) and 0 < f(2000, n, m, 0, 0) < f(2000, n, m, count, rank)
    g = L.hscale_adapted_linear_grad_workspace_bytes
    assert g(0, n, m, count, rank) == g(T, n, m, 0, rank) == g(T, 24, m, count, rank) == 0
    assert g(T, n, m, count, rank) > 0
    for h in (L.hscale_token_loss_workspace_bytes, L.hscale_token_loss_grad_workspace_bytes):
        assert h(0, 64, 10) == h(4, 24, 10) == h(4, 64, 0) == h(1 << 20, 64, 1 << 20) == 0
        assert h(4, 64, 10) > 0
    # what holds g is bounded: a large vocabulary is taken in pieces
    big = L.hscale_token_loss_grad_workspace_bytes(8192, 4096, 128000)
    assert big <= (512 << 20) + 8192 * 4096 * 4 + 8192 * 4096 * 2 + 1024


def test_adapted_linear_refusals(L):
    need = L.hscale_adapted_linear_workspace_bytes(T, n, m, count, rank)

    def call(**k):
        g = lambda name, default: k.get(name, default)  # noqa: E731
        return L.hscale_adapted_linear(g("X", A), g("T", T), g("n", n), g("ldx", n), g("m", m), g("s", 1e-3),
                                       g("codes", 2 * A), g("packed", 3 * A), g("ad", AD), g("Y", 4 * A),
                                       g("ldy", m), g("ws", 5 * A), g("wsb", need), 0)

    def ad(**k):
        names = ("count", "rank", "A", "B", "alpha", "adapter")
        return call(ad=tuple(k.get(a, v) for a, v in zip(names, AD)))

    assert call(T=0, X=0, Y=0, ws=0) == 0 and call(m=0, ldy=0) == 0
    assert call(n=24) == call(T=-1) == call(m=-1) == call(n=0) == -2
    assert call(T=(1 << 24) + 1) == call(n=(1 << 21) + 16) == call(m=(1 << 21) + 1) == -2
    assert call(ldx=n - 16) == call(ldx=(1 << 21) + 16) == call(ldy=m - 1) == -2
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert call(s=s) == -5
    for name in ("X", "codes", "packed", "Y", "ws"):
        assert call(**{name: 0}) == -1, name
    assert call(X=A + 8) == call(ldx=n + 4) == call(packed=3 * A + 4) == call(Y=4 * A + 1) == call(ws=5 * A + 8) == -3
    assert call(wsb=need - 1) == -6
    assert call(Y=A + 64) == call(Y=2 * A) == call(Y=3 * A) == call(ws=4 * A) == call(Y=10 * A) == call(Y=13 * A) == -8
    assert ad(count=-1) == ad(count=4097) == ad(rank=0) == ad(rank=12) == ad(rank=264) == -2
    assert ad(A=0) == ad(B=0) == -1
    assert ad(A=10 * A + 8) == ad(B=11 * A + 2) == ad(alpha=12 * A + 2) == ad(adapter=13 * A + 2) == -3


def test_checkpoint_refusals(L):
    def pack(**k):
        g = lambda name, default: k.get(name, default)  # noqa: E731
        return L.hscale_pack_activations(g("X", A), g("T", T), g("n", n), g("ldx", n), g("q", 2 * A), g("s", 3 * A), 0)

    def unpack(**k):
        g = lambda name, default: k.get(name, default)  # noqa: E731
        return L.hscale_unpack_activations(g("q", 2 * A), g("s", 3 * A), g("T", T), g("n", n), g("X", A),
                                           g("ldx", n), 0)

    for f in (pack, unpack):
        assert f(T=0) == f(n=0) == 0
        assert f(n=20) == f(T=-1) == f(ldx=n - 1) == -2
        assert f(X=0) == f(q=0) == f(s=0) == -1
        assert f(q=2 * A + 4) == f(s=3 * A + 1) == f(X=A + 1) == -3
        assert f(q=A) == f(s=A + 4) == -8
    assert pack(ldx=n + 4) == pack(X=A + 8) == -3
    assert pack(s=2 * A) == -8


def test_adapted_linear_grad_refusals(L):
    need = L.hscale_adapted_linear_grad_workspace_bytes(T, n, m, count, rank)

    def call(**k):
        g = lambda name, default: k.get(name, default)  # noqa: E731
        return L.hscale_adapted_linear_grad(g("dY", A), g("T", T), g("m", m), g("lddy", m), g("q", 2 * A),
                                            g("s", 3 * A), g("n", n), g("sg", 1e-3), g("codes", 4 * A),
                                            g("packed", 5 * A), g("ad", AD), g("dX", 6 * A), g("lddx", n),
                                            g("dA", 7 * A), g("dB", 8 * A), g("ws", 9 * A), g("wsb", need), 0)

    assert call(n=24) == call(T=-1) == call(n=0) == call(m=0) == call(lddy=m - 1) == call(lddx=n - 1) == -2
    assert call(ad=None) == -1 and call(ad=(0, 8, A, A, 0, 0)) == -2
    assert call(sg=0.0) == -5
    for name in ("dY", "q", "s", "codes", "packed", "dA", "dB", "ws"):
        assert call(**{name: 0}) == -1, name
    assert call(dY=A + 1) == call(q=2 * A + 4) == call(dX=6 * A + 1) == call(dA=7 * A + 1) == call(ws=9 * A + 16) == -3
    assert call(wsb=need // 2) == -6
    assert call(dX=A) == call(dA=10 * A) == call(dB=7 * A) == call(ws=2 * A) == call(dB=11 * A) == -8


def test_token_loss_refusals(L):
    V = 50
    need, need_grad = (f(T, n, V) for f in (L.hscale_token_loss_workspace_bytes,
                                            L.hscale_token_loss_grad_workspace_bytes))

    def loss(**k):
        g = lambda name, default: k.get(name, default)  # noqa: E731
        return L.hscale_token_loss(g("X", A), g("T", T), g("n", n), g("ldx", n), g("W", 2 * A), g("V", V),
                                   g("y", 3 * A), g("loss", 4 * A), g("lse", 5 * A), g("ws", 6 * A), g("wsb", need), 0)

    def grad(**k):
        g = lambda name, default: k.get(name, default)  # noqa: E731
        return L.hscale_token_loss_grad(g("X", A), g("T", T), g("n", n), g("ldx", n), g("W", 2 * A), g("V", V),
                                        g("y", 3 * A), g("lse", 5 * A), g("w", 7 * A), g("dX", 8 * A), g("lddx", n),
                                        g("dW", 9 * A), g("ws", 6 * A), g("wsb", need_grad), 0)

    for f in (loss, grad):
        assert f(n=24) == f(T=-1) == f(V=0) == f(n=0) == f(ldx=n - 8) == f(V=(1 << 24) + 1) == f(V=-1) == -2
        assert f(X=0) == f(W=0) == f(y=0) == f(lse=0) == f(ws=0) == -1
        assert f(X=A + 2) == f(ldx=n + 4) == f(W=2 * A + 8) == f(y=3 * A + 4) == f(ws=6 * A + 128) == -3
        assert f(wsb=need // 4) == -6
        assert f(ws=A) == -8
    assert loss(T=0) == 0 and loss(loss=0) == -1 and loss(loss=3 * A) == loss(lse=4 * A) == -8
    assert grad(T=0, dW=0) == 0 and grad(w=0) == -1
    assert grad(dX=8 * A + 4) == grad(lddx=n + 2) == grad(dW=9 * A + 4) == grad(w=7 * A + 2) == -3
    assert grad(dX=A) == grad(dW=2 * A) == grad(dX=9 * A) == grad(dW=7 * A) == -8


# ---------------------------------------------------------------------------
# The torch front end
# ---------------------------------------------------------------------------


def i32(*s):
    return torch.empty(s, dtype=torch.int32, device="meta")


def i64(*s):
    return torch.empty(s, dtype=torch.int64, device="meta")


def _layer():
    return dict(global_scale=1e-3, scale_codes=u8(m, n // 16), packed_e2m1=u8(m, n // 2))


def _low():
    return dict(A=bf(count, rank, n), B=bf(count, m, rank), alpha=f32(count), adapter=i32(T))


def short(t):
    return t[:-1]


ALL = (on_host, wrong_dtype, one_more_row, strided)
ROWS = (on_host, wrong_dtype, strided, one_more_row)  # any row stride, unit column stride
CASES = {
    "adapted_linear": (ops.adapted_linear, lambda: dict(X=bf(T, 2 * n)[:, :n], **_layer(), **_low(),
                                                        Y=bf(T, m + 3)[:, :m], workspace=u8(64)),
                       dict(X=(on_host, wrong_dtype, strided, flat, short), scale_codes=ALL, packed_e2m1=ALL, A=ALL,
                            B=ALL + (short,), alpha=ALL, adapter=ALL + (short,), Y=ROWS, workspace=SCRATCH)),
    "pack_activations": (ops.pack_activations, lambda: dict(X=bf(T, 2 * n)[:, :n], q=i8(T, n), scale=f32(T, 1)),
                         dict(X=(on_host, wrong_dtype, strided, flat), q=ALL, scale=ALL[:3])),
    "unpack_activations": (ops.unpack_activations, lambda: dict(q=i8(T, n), scale=f32(T, 1), X=bf(T, n + 1)[:, :n]),
                           dict(q=(on_host, wrong_dtype, strided, flat, short), scale=ALL[:3], X=ROWS)),
    "adapted_linear_grad": (ops.adapted_linear_grad,
                            lambda: dict(dY=bf(T, m + 5)[:, :m], q=i8(T, n), scale=f32(T, 1), **_layer(), **_low(),
                                         dX=bf(T, n + 1)[:, :n], dA=bf(count, rank, n), dB=bf(count, m, rank),
                                         workspace=u8(64)),
                            dict(dY=(on_host, wrong_dtype, strided, flat, short), q=ALL, scale=ALL[:3],
                                 scale_codes=ALL, packed_e2m1=ALL, A=ALL, B=ALL, alpha=ALL, adapter=ALL, dX=ROWS,
                                 dA=ALL, dB=ALL, workspace=SCRATCH)),
    "token_loss": (ops.token_loss, lambda: dict(X=bf(T, 2 * n)[:, :n], W=bf(50, n), target=i64(T), loss=f32(T),
                                                lse=f32(T), workspace=u8(64)),
                   dict(X=(on_host, wrong_dtype, strided, flat, short), W=(on_host, wrong_dtype, strided, flat),
                        target=ALL, loss=ALL, lse=ALL, workspace=SCRATCH)),
    "token_loss_grad": (ops.token_loss_grad,
                        lambda: dict(X=bf(T, 2 * n)[:, :n], W=bf(50, n), target=i64(T), lse=f32(T), weight=f32(T),
                                     dX=bf(T, n + 1)[:, :n], dW=bf(50, n), workspace=u8(64)),
                        dict(X=(on_host, wrong_dtype, strided, flat, short), W=(on_host, wrong_dtype, strided, flat),
                             target=ALL, lse=ALL, weight=ALL, dX=ROWS, dW=ALL, workspace=SCRATCH)),
}
BAD = [(fn, arg, mut) for fn, (_, _, args) in CASES.items() for arg, muts in args.items() for mut in muts]


@pytest.mark.parametrize("fn", sorted(CASES))
def test_good_buffers_reach_the_library(fake_gpu, fn):  # noqa: F811
    f, good, _ = CASES[fn]
    with pytest.raises(Reached):
        f(**good(), stream=0)


@pytest.mark.parametrize("fn,arg,mutation", BAD, ids=lambda v: getattr(v, "__name__", v))
def test_bad_buffer_refused_before_the_library(fake_gpu, fn, arg, mutation):  # noqa: F811
    f, good, _ = CASES[fn]
    kwargs = good()
    kwargs[arg] = mutation(kwargs[arg])
    with pytest.raises(ValueError):
        f(**kwargs, stream=0)


def test_adapters_given_in_part_are_refused(fake_gpu):  # noqa: F811
    X, layer, low = bf(T, n), _layer(), _low()
    for given in (dict(A=low["A"]), dict(B=low["B"]), dict(alpha=low["alpha"]), dict(adapter=low["adapter"]),
                  dict(A=low["A"], B=low["B"])):  # three adapters, and no tokens' numbers
        with pytest.raises(ValueError):
            ops.adapted_linear(X, **layer, **given, stream=0)
    with pytest.raises(ValueError):
        ops.adapted_linear_grad(bf(T, m), i8(T, n), f32(T, 1), **layer, A=None, B=None, stream=0)
    with pytest.raises(ValueError):
        ops.adapted_linear_grad(bf(T, m), i8(T, n), f32(T, 1), **layer, **low, dX=bf(T, n), need_dX=False, stream=0)
    with pytest.raises(ValueError):
        ops.token_loss_grad(X, bf(50, n), i64(T), f32(T), f32(T), dW=bf(50, n), need_dW=False, stream=0)


# ---------------------------------------------------------------------------
# The kernels as compiled
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("source", ["adapt.hip", "loss.hip"])
def test_no_kernel_uses_scratch(tmp_path, source):
    csrc = ROOT / "paper_2608_28113_amd" / "csrc"
    asm = tmp_path / "out.s"
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    r = subprocess.run([build.HIPCC, *flags, "--cuda-device-only", "-S", "-I", str(ROOT / "include"), "-I", str(csrc),
                        "-o", str(asm), str(csrc / source)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    used = {k: int(v) for k, v in re.findall(r"^\s+\.set (\S+)\.private_seg_size, (\d+)", asm.read_text(), re.M)}
    assert used and not {k: v for k, v in used.items() if v}, used
