"""Refusals of routing, the layer of stored experts and the rules on logits: at
the C ABI (fake addresses; nothing here reaches the HIP runtime) and in the
torch front end (`meta` tensors, and stubs that no bad buffer may reach)."""
import os
import re
import subprocess
from pathlib import Path

import pytest
import torch

from paper_2608_28113_amd import _lib, build, ops
from tests.test_front_end import (SCRATCH, Reached, bf, f32, fake_gpu, flat, on_host,  # noqa: F401
                                  one_more_row, strided, u8, wrong_dtype)

ROOT = Path(__file__).resolve().parent.parent
A = 1 << 34  # fake but aligned device addresses, far apart
T, n, hidden, E, k = 100, 64, 48, 5, 2
R, V, L = 6, 100, 20


@pytest.fixture(scope="module")
def lib():
    if not _lib.LIB_PATH.exists():
        build.build()
    _lib.load()
    return _lib


def test_route_refusals(lib):
    def call(**a):
        g = lambda name, default: a.get(name, default)  # noqa: E731
        return lib.hscale_route_tokens(g("logits", A), g("type", 0), g("T", T), g("E", E), g("ld", E), g("k", k), 1,
                                       g("expert", 2 * A), g("weight", 3 * A), 0)

    assert call(T=0, logits=0) == 0
    assert call(T=-1) == call(T=(1 << 24) + 1) == call(E=0) == call(E=1025) == call(ld=E - 1) == -2
    assert call(k=0) == call(k=E + 1) == call(E=64, ld=64, k=33) == call(type=2) == call(type=-1) == -2
    for name in ("logits", "expert", "weight"):
        assert call(**{name: 0}) == -1, name
    assert call(logits=A + 1) == call(logits=A + 2, type=1) == call(expert=2 * A + 2) == call(weight=3 * A + 1) == -3
    assert call(weight=2 * A) == call(expert=A) == call(weight=A + 16) == -8


def test_expert_workspace(lib):
    f = lib.hscale_expert_layer_workspace_bytes
    assert f(0, n, hidden, E, k) == f(T, 0, hidden, E, k) == f(T, n, 0, E, k) == 0
    assert f(T, 24, hidden, E, k) == f(T, n, 24, E, k) == f(-1, n, hidden, E, k) == f((1 << 24) + 1, n, hidden, E, k) == 0
    assert f(T, n, hidden, 0, k) == f(T, n, hidden, 1025, k) == f(T, n, hidden, E, 0) == f(T, n, hidden, E, 33) == 0
    for sizes in ((4096, 14336, 8, 2), (64, 48, 5, 2), (2048, 1024, 64, 32), (1 << 21, 1 << 21, 3, 32)):
        at = [f(t, *sizes) for t in (1, 2, 3, 16, 17, 100, 127, 128, 129, 511, 512, 2048, 2049, 4097, 100000, 1 << 24)]
        assert at[0] > 0 and at == sorted(at), sizes
    # longer calls go in pieces
    assert f(1 << 24, 4096, 14336, 8, 2) == f(2048, 4096, 14336, 8, 2)


def test_expert_layer_refusals(lib):
    need = lib.hscale_expert_layer_workspace_bytes(T, n, hidden, E, k)
    names = ("gate", "up", "down")

    def call(**a):
        g = lambda name, default: a.get(name, default)  # noqa: E731
        m = [g(name, (10 * i * A, (10 * i + 1) * A, (10 * i + 2) * A)) for i, name in enumerate(names, 2)]
        return lib.hscale_expert_layer(g("X", A), g("T", T), g("n", n), g("ldx", n), g("hidden", hidden), g("E", E), *m,
                                       g("expert", 2 * A), g("weight", 3 * A), g("k", k), g("Y", 4 * A), g("ldy", n),
                                       g("ws", 5 * A), g("wsb", need), 0)

    assert call(T=0, X=0, gate=None) == 0
    assert call(T=-1) == call(T=(1 << 24) + 1) == call(n=24) == call(n=0) == call(hidden=0) == call(hidden=40) == -2
    assert call(n=(1 << 21) + 16) == call(hidden=(1 << 21) + 16) == call(E=0) == call(E=1025) == -2
    assert call(k=0) == call(k=33) == call(ldx=n - 1) == call(ldx=(1 << 21) + 8) == call(ldy=n - 1) == -2
    for name in ("X", "expert", "weight", "Y", "ws"):
        assert call(**{name: 0}) == -1, name
    for name in names:
        good = (10 * A, 11 * A, 12 * A)
        assert call(**{name: None}) == -1
        for i in range(3):
            assert call(**{name: tuple(0 if j == i else v for j, v in enumerate(good))}) == -1
        assert call(**{name: (10 * A + 2, 11 * A, 12 * A)}) == call(**{name: (10 * A, 11 * A, 12 * A + 4)}) == -3
        for at in good:  # results over a matrix
            assert call(**{name: good, "Y": at}) == call(**{name: good, "ws": at}) == -8
    assert call(X=A + 8) == call(ldx=n + 4) == call(Y=4 * A + 1) == call(ws=5 * A + 128) == -3
    assert call(expert=2 * A + 2) == call(weight=3 * A + 1) == -3
    assert call(wsb=need - 1) == call(wsb=0) == -6
    assert call(Y=A) == call(Y=2 * A) == call(Y=3 * A) == call(Y=5 * A + 256) == call(ws=A) == call(ws=3 * A) == -8


FIELDS = dict(history=10 * A, history_length=L, history_ld=L, length=11 * A, prompt=12 * A, repetition=13 * A,
              frequency=14 * A, presence=15 * A, bias=16 * A, biases=2, bias_row=17 * A, mask=18 * A, masks=3,
              mask_row=19 * A)


def test_adjust_refusals(lib):
    def call(**a):
        g = lambda name, default: a.get(name, default)  # noqa: E731
        rules = None if "rules" in a else tuple(a.get(f, v) for f, v in FIELDS.items())
        return lib.hscale_adjust_logits(rules, g("logits", A), g("type", 0), g("R", R), g("V", V), g("ld", V),
                                        g("out", 2 * A), g("ldo", V), 0)

    assert call(R=0, logits=0) == call(V=0, out=0) == 0
    assert call(rules=None) == -1
    assert call(R=-1) == call(V=-1) == call(R=(1 << 24) + 1) == call(V=(1 << 24) + 1) == call(type=2) == -2
    assert call(ld=V - 1) == call(ldo=V - 1) == call(history_length=-1) == call(history_ld=L - 1) == -2
    assert call(history_length=(1 << 30) + 1, history_ld=1 << 31) == -2
    assert call(biases=-1) == call(masks=-1) == call(bias_row=0) == call(mask_row=0) == -2  # two biases, three masks
    assert call(biases=(1 << 24) + 1) == call(masks=(1 << 24) + 1) == -2
    assert call(logits=0) == call(out=0) == call(history=0) == -1
    assert call(logits=A + 1) == call(out=2 * A + 1) == call(logits=A + 2, type=1) == call(out=2 * A + 2, type=1) == -3
    for f, v in FIELDS.items():
        if v >= A:
            assert call(**{f: v + 2}) == -3, f
            assert call(out=v) == -8, f
    assert call(out=A + 2) == call(out=A, ldo=V + 1) == call(logits=A + 2 * V, out=A) == -8


# ---------------------------------------------------------------------------
# The torch front end
# ---------------------------------------------------------------------------


def i32(*s):
    return torch.empty(s, dtype=torch.int32, device="meta")


def short(t):
    return t[:-1]


def _stored(rows, cols):
    return dict(s=f32(E), c=u8(E, rows, cols // 16), p=u8(E, rows, cols // 2))


def _layer(X, expert, weight, Y, workspace, **m):
    gate, up, down = (tuple(m[a + f] for f in "scp") for a in ("g", "u", "d"))
    return ops.expert_layer(X, expert, weight, gate, up, down, Y=Y, workspace=workspace, stream=0)


def _layer_args():
    args = dict(X=bf(T, 2 * n)[:, :n], expert=i32(T, k), weight=f32(T, k), Y=bf(T, n + 3)[:, :n], workspace=u8(64))
    for a, m in (("g", _stored(hidden, n)), ("u", _stored(hidden, n)), ("d", _stored(n, hidden))):
        args.update({a + f: v for f, v in m.items()})
    return args


def _adjust_args():
    return dict(logits=bf(R, V + 3)[:, :V], history=i32(R, L + 4)[:, :L], length=i32(R), prompt=i32(R),
                repetition=f32(R), frequency=f32(R), presence=f32(R), bias=f32(2, V), bias_row=i32(R),
                mask=i32(3, -(-V // 32)), mask_row=i32(R), out=bf(R, V + 1)[:, :V])


def half(t):
    return torch.empty(t.shape, dtype=torch.float16, device=t.device)


ALL = (on_host, wrong_dtype, one_more_row, strided, short)
ROWS = (on_host, wrong_dtype, strided, one_more_row, flat)
SET = (on_host, wrong_dtype, strided, flat)  # any number of biases, masks
CASES = {
    "route_tokens": (lambda **a: ops.route_tokens(a.pop("logits"), k, **a, stream=0),
                     lambda: dict(logits=bf(T, E + 3)[:, :E], expert=i32(T, k), weight=f32(T, k)),
                     dict(logits=(on_host, half, strided, flat, short), expert=ALL, weight=ALL)),
    "expert_layer": (_layer, _layer_args,
                     dict(X=(on_host, wrong_dtype, strided, flat, short), expert=ALL + (flat,), weight=ALL, Y=ROWS,
                          workspace=SCRATCH, **{a + f: ALL for a in "gud" for f in "scp"})),
    "adjust_logits": (lambda **a: ops.adjust_logits(**a, stream=0), _adjust_args,
                      dict(logits=(on_host, half, strided, flat, short), history=ROWS, length=ALL, prompt=ALL,
                           repetition=ALL, frequency=ALL, presence=ALL, bias=SET, bias_row=ALL, mask=SET, mask_row=ALL,
                           out=ROWS)),
}
BAD = [(fn, arg, mut) for fn, (_, _, args) in CASES.items() for arg, muts in args.items() for mut in muts]


@pytest.mark.parametrize("fn", sorted(CASES))
def test_good_buffers_reach_the_library(fake_gpu, fn):  # noqa: F811
    f, good, _ = CASES[fn]
    with pytest.raises(Reached):
        f(**good())


@pytest.mark.parametrize("fn,arg,mutation", BAD, ids=lambda v: getattr(v, "__name__", v))
def test_bad_buffer_refused_before_the_library(fake_gpu, fn, arg, mutation):  # noqa: F811
    f, good, _ = CASES[fn]
    kwargs = good()
    kwargs[arg] = mutation(kwargs[arg])
    with pytest.raises(ValueError):
        f(**kwargs)


@pytest.mark.parametrize("bad", [0, -1, E + 1])
def test_choices_out_of_range(fake_gpu, bad):  # noqa: F811
    with pytest.raises(ValueError):
        ops.route_tokens(bf(T, E), bad, stream=0)


def test_rules_given_in_part_are_refused(fake_gpu):  # noqa: F811
    a = _adjust_args()
    for names in (("length",), ("prompt",), ("repetition",), ("frequency",), ("presence",), ("bias_row",),
                  ("mask_row",), ("bias",), ("mask",)):  # two biases, three masks and no rows' numbers
        with pytest.raises(ValueError):
            ops.adjust_logits(a["logits"], **{x: a[x] for x in names}, stream=0)


def test_matrices_of_other_shapes_are_refused(fake_gpu):  # noqa: F811
    a = _layer_args()
    gate, up, down = (tuple(a[m + f] for f in "scp") for m in "gud")
    for m in ((down, up, down), (gate, down, down), (gate, up, gate), (gate[:2], up, down), (None, up, down)):
        with pytest.raises(ValueError):
            ops.expert_layer(a["X"], a["expert"], a["weight"], *m, stream=0)


@pytest.mark.parametrize("fn,arg", [("route_tokens", "logits"), ("expert_layer", "X"), ("expert_layer", "weight")]
                         + [("adjust_logits", a) for a in ("logits", "repetition", "frequency", "presence", "bias")])
def test_a_graph_that_is_not_recorded_is_refused(fake_gpu, fn, arg):  # noqa: F811
    f, good, _ = CASES[fn]
    kwargs = good()
    kwargs[arg] = kwargs[arg].detach().requires_grad_()
    with pytest.raises(ValueError, match="no_grad"):
        f(**kwargs)
    with torch.no_grad(), pytest.raises(Reached):
        f(**kwargs)


# ---------------------------------------------------------------------------
# The code as compiled
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("source", ["experts.hip", "logits.hip"])
def test_no_kernel_uses_scratch(tmp_path, source):
    csrc = ROOT / "paper_2608_28113_amd" / "csrc"
    asm = tmp_path / "out.s"
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    r = subprocess.run([build.HIPCC, *flags, "--cuda-device-only", "-S", "-I", str(ROOT / "include"), "-I", str(csrc),
                        "-o", str(asm), str(csrc / source)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    used = {name: int(v) for name, v in re.findall(r"^\s+\.set (\S+)\.private_seg_size, (\d+)", asm.read_text(), re.M)}
    assert used and not {name: v for name, v in used.items() if v}, used


@pytest.mark.skipif(not Path(build.HIPCC).exists(), reason="hipcc not installed")
def test_host_code_is_sanitizer_clean(tmp_path):
    """Plans and validation under AddressSanitizer and UndefinedBehaviorSanitizer
    (the host's code only; nothing is launched)."""
    csrc = ROOT / "paper_2608_28113_amd" / "csrc"
    common = [build.HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-ffp-contract=off",
              "-fhip-fp32-correctly-rounded-divide-sqrt", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
              "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
              "-Xarch_host", "-fno-omit-frame-pointer", "-I", str(ROOT / "include"), "-I", str(csrc)]
    units = [(csrc / f"{u}.hip", tmp_path / f"{u}.o") for u in ("experts", "logits")]
    units.append((ROOT / "tests" / "native" / "decode_sanitize_driver.cpp", tmp_path / "driver.o"))
    exe = tmp_path / "driver"
    for src, obj in units:
        r = subprocess.run(common + ["-x", "hip", "-c", "-o", str(obj), str(src)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([build.HIPCC, "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address",
                        "-Xarch_host", "-fsanitize=undefined", "-o", str(exe), *[str(o) for _, o in units], "-lm"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "sanitize driver: ok" in r.stdout, (r.stdout + r.stderr)[-3000:]
