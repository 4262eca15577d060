"""Memory that the torch front end allocates for a call on another stream than
the current one (CPU only: 'meta' tensors stand in for device tensors, and the
streams are stand-ins).  The allocator gives memory out again in the order of
the stream it was allocated on: outputs and scratch of a call on a side stream
that came from the current stream's pool could still be in use there, and
scratch would go back to it while the call runs."""
import contextlib
import gc
import weakref

import pytest
import torch

from paper_2608_28113_amd import _lib, ops
from tests.test_adapt_abi import CASES as ADAPT
from tests.test_front_end import CASES as BASE
from tests.test_front_end import Reached, fake_gpu  # noqa: F401

SIDE, HERE = object(), object()
CASES = {**BASE, **ADAPT}
# what a call may allocate: its optional outputs and scratch
GIVEN = ("h", "scale_codes", "packed_e2m1", "workspace", "row_err", "Y", "q", "scale", "dX", "dA", "dB", "loss", "lse",
         "dW", "X")
KEEP = {"search_block": GIVEN, "quantize": ("scale_codes",), "output_error": ("scale_codes", "packed_e2m1", "X"),
        "adapted_linear": ("scale_codes", "packed_e2m1", "X"), "hdiag": ("X",), "hdiag_accumulate": ("X",),
        "search": ("h",), "search_stats": ("h",), "pack_activations": ("X",), "unpack_activations": ("q", "scale"),
        "adapted_linear_grad": ("q", "scale", "scale_codes", "packed_e2m1"), "token_loss": ("X",),
        "token_loss_grad": ("X", "lse")}


@pytest.fixture
def allocations(fake_gpu, monkeypatch):  # noqa: F811
    """[(shape, the stream it was allocated under, the stream it was recorded on)]."""
    made, under = [], [HERE]

    @contextlib.contextmanager
    def stream(s):
        under.append(s)
        yield
        under.pop()

    def watch(make):
        def f(*shape, **kw):
            before = len(made)
            t = make(*shape, **kw)
            made[before:] = [[t, under[-1], None]]  # not those that make() makes in turn
            return t
        return f

    def record(t, s):
        for m in made:
            if m[0] is t:
                m[2] = s

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: HERE)
    monkeypatch.setattr(torch.Tensor, "record_stream", record)
    monkeypatch.setattr(ops, "_elsewhere", lambda s, device: s if s is SIDE else None, raising=False)
    monkeypatch.setattr(ops, "_stream", lambda s, device: 0)
    monkeypatch.setattr(torch, "empty", watch(torch.empty))
    monkeypatch.setattr(torch, "zeros", watch(torch.zeros))
    return made


def _arguments(fn):
    f, good, _ = CASES[fn]
    given = good()
    return f, {k: v for k, v in given.items() if k not in GIVEN or k in KEEP.get(fn, ())}


def _call(fn, made, stream):
    f, given = _arguments(fn)
    del made[:]  # the arguments' own
    with pytest.raises(Reached):
        f(**given, stream=stream)


@pytest.mark.parametrize("fn", sorted(CASES))
def test_new_memory_belongs_to_the_stream_of_the_call(allocations, fn):
    _call(fn, allocations, SIDE)
    assert allocations or fn in ("search_block", "hdiag_finalize")
    for t, under, recorded in allocations:
        assert under is SIDE, (fn, t.shape)
        scratch = t.dtype is torch.uint8 and t.dim() == 1
        assert recorded is (None if scratch else HERE), (fn, t.shape)


@pytest.mark.parametrize("fn", sorted(CASES))
def test_on_the_current_stream_nothing_is_recorded(allocations, fn):
    _call(fn, allocations, None)
    assert all(under is HERE and recorded is None for _, under, recorded in allocations)


@pytest.mark.parametrize("fn", ["hdiag", "output_error", "adapted_linear", "adapted_linear_grad", "token_loss",
                                "token_loss_grad"])
def test_scratch_lives_until_the_library_was_called(fake_gpu, monkeypatch, fn):  # noqa: F811
    """Freed before, it could be given to another thread ahead of the launches."""
    f, given = _arguments(fn)
    scratch, empty = [], torch.empty

    def watch(*shape, **kw):
        t = empty(*shape, **kw)
        if t.dtype is torch.uint8 and t.dim() == 1:
            scratch.append(weakref.ref(t))
        return t

    def reached(*args):
        gc.collect()
        assert scratch and all(r() is not None for r in scratch)
        raise Reached

    monkeypatch.setattr(torch, "empty", watch)
    monkeypatch.setattr(_lib, f"hscale_{fn}", reached)
    with pytest.raises(Reached):
        f(**given, stream=0)


def test_a_stream_is_another_one_by_its_handle(monkeypatch):
    device = torch.device("cuda", 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 48, raising=False)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device: ("external", handle))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device: "default")
    assert ops._elsewhere(None, device) is None and ops._elsewhere(48, device) is None
    assert ops._elsewhere(64, device) == ("external", 64) and ops._elsewhere(0, device) == "default"
    assert ops._elsewhere(64, torch.device("meta")) is None
