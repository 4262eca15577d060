"""Penalties, biases and masks on logits against a 64-bit plain implementation."""
from __future__ import annotations

import pytest
import torch

from tests import decode_ref as ref

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"
BOTH = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    yield hs
    torch.cuda.empty_cache()  # what is cached here would serve later tests that bound the memory left


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _rules(R, V, L, biases, masks, seed=0):
    """Histories with words outside the vocabulary, lengths and prompts outside
    theirs, numbers that mean no bias and no mask, and a mask that leaves nothing."""
    g = _gen(seed)
    few = torch.randint(0, V, (max(1, V // 7),), generator=g)
    p = dict(history=few[torch.randint(0, len(few), (R, L), generator=g)].int(),
             length=torch.randint(-2, L + 3, (R,), generator=g, dtype=torch.int32),
             prompt=torch.randint(-1, L + 2, (R,), generator=g, dtype=torch.int32),
             repetition=0.7 + torch.rand(R, generator=g), frequency=torch.randn(R, generator=g),
             presence=torch.randn(R, generator=g))
    p["history"][torch.rand((R, L), generator=g) < 0.1] = -1
    p["history"][torch.rand((R, L), generator=g) < 0.1] = V
    if biases:
        p["bias"] = torch.randn((biases, V), generator=g)
        p["bias_row"] = torch.randint(-1, biases + 1, (R,), generator=g, dtype=torch.int32)
    if masks:
        p["mask"] = torch.randint(-2 ** 31, 2 ** 31, (masks, -(-V // 32)), generator=g).int()
        p["mask"][0] = 0
        p["mask_row"] = torch.randint(-1, masks + 1, (R,), generator=g, dtype=torch.int32)
    return {k: v.to(DEV) for k, v in p.items()}


def _close(got, want, size):
    """Each of five steps in fp32 errs by at most 2^-24 of a term or a sum of
    them, all within `size`, and the result is rounded by half a step of its
    type: 2^-8 or 2^-24 of it.  What is past the type's range by a whole step or
    more is infinite in it: the lowest value times 1.25 is -inf."""
    got = got.cpu()
    end = torch.finfo(got.dtype)
    want = torch.where(want.abs() >= end.max * (1.0 + end.eps), want * float("inf"), want)
    last = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    got, finite = got.double(), want.isfinite()
    assert torch.equal(got.isfinite(), finite) and torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got[~finite & ~want.isnan()], want[~finite & ~want.isnan()])
    worst = ((got - want).abs() - last * want.abs() - 5 * 2.0 ** -24 * size)[finite]
    assert not worst.numel() or worst.max() <= 0.0


@pytest.mark.parametrize("R,V,L", [(1, 1, 1), (1, 7, 3), (3, 33, 40), (2, 2048, 100), (5, 2049, 1025), (2, 8200, 5),
                                   (1, 4099, 3001), (300, 100, 17)])
@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("biases,masks", [(0, 0), (2, 3)])
def test_rules(hs, R, V, L, dtype, biases, masks):
    logits = (torch.randn((R, V), generator=_gen(V)) * 3).to(dtype).to(DEV)
    p = _rules(R, V, L, biases, masks, seed=R)
    print(f"[logits {R} {V} {L}]", flush=True)
    _close(hs.adjust_logits(logits, **p), *ref.logits(logits, **p))


@pytest.mark.parametrize("names", [("history", "repetition"), ("history", "length", "frequency"),
                                   ("history", "prompt", "presence"), ("bias", "bias_row"), ("mask", "mask_row"),
                                   ("history", "mask", "mask_row"), ()])
@pytest.mark.parametrize("dtype", BOTH)
def test_each_rule_alone(hs, names, dtype):
    logits = torch.randn((6, 301), generator=_gen(1)).to(dtype).to(DEV)
    p = _rules(6, 301, 50, 3, 4)
    p = {k: p[k] for k in names}
    got = hs.adjust_logits(logits, **p)
    _close(got, *ref.logits(logits, **p))
    if not names:
        assert torch.equal(got, logits)


def test_one_bias_and_one_mask_for_all(hs):
    logits = torch.randn((4, 90), generator=_gen(1)).to(DEV)
    p = _rules(4, 90, 8, 1, 1)
    p["mask"].fill_(0x5A5A5A5A)
    p = dict(bias=p["bias"], mask=p["mask"])
    _close(hs.adjust_logits(logits, **p), *ref.logits(logits, **p))


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("R,V", [(3, 77), (2, 70001)])
def test_in_place_and_strided(hs, dtype, R, V):
    big = torch.full((R + 1, V + 9), 5.0, dtype=dtype, device=DEV)
    view = big[:R, 3:3 + V]
    view.copy_(torch.randn((R, V), generator=_gen(1)))
    logits = view.clone()
    p = _rules(R, V, 60, 2, 2)
    if V < 1000:
        want = ref.logits(logits, **p)
    else:
        out = hs.adjust_logits(logits, **p)
    other = torch.full((R + 1, V + 5), 4.0, dtype=dtype, device=DEV)
    got = hs.adjust_logits(view, **p, out=other[:R, 1:1 + V])
    assert hs.adjust_logits(view, **p, out=view) is view
    assert torch.equal(view, got)
    if V < 1000:
        _close(got, *want)
    else:
        assert torch.equal(got, out)
    view.fill_(5.0)
    got.fill_(4.0)
    assert (big == 5.0).all() and (other == 4.0).all()
    wide = torch.full((R, 80), -9, dtype=torch.int32, device=DEV)  # a history with strided rows
    wide[:, 5:65] = p["history"]
    p["history"] = wide[:, 5:65]
    again = hs.adjust_logits(logits, **p)
    if V < 1000:
        _close(again, *want)
    else:
        assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", BOTH)
def test_what_is_not_finite(hs, dtype):
    """Infinities and NaN in logits stay in their place, masked ones go, and a
    row that the mask leaves nothing is all -inf."""
    inf, nan = float("inf"), float("nan")
    low = torch.finfo(dtype).min
    logits = torch.tensor([[inf, -inf, nan, low, 1.0, 0.0, -0.0, 2.0]] * 4).to(dtype).to(DEV)
    history = torch.tensor([[0, 1, 2, 3, 4, 5, 6, 7]] * 4, dtype=torch.int32, device=DEV)
    p = dict(history=history, repetition=torch.full((4,), 1.25, device=DEV), frequency=torch.full((4,), 0.5, device=DEV),
             presence=torch.full((4,), -0.25, device=DEV),
             mask=torch.tensor([[0], [0b11111000], [0b00000111]], dtype=torch.int32, device=DEV),
             mask_row=torch.tensor([0, 1, 2, -1], dtype=torch.int32, device=DEV))
    got = hs.adjust_logits(logits, **p)
    assert torch.isneginf(got[0]).all()
    assert torch.isneginf(got[1, :3]).all() and got[2, 2].isnan() and torch.isneginf(got[2, 3:]).all()
    _close(got, *ref.logits(logits, **p))


def test_no_rows_no_words_no_history(hs):
    p = _rules(3, 40, 5, 0, 0)
    logits = torch.randn((3, 40), device=DEV)
    none = {k: v[:0] for k, v in p.items()}
    assert hs.adjust_logits(logits[:0], **none).shape == (0, 40)
    assert hs.adjust_logits(logits[:, :0], **p).shape == (3, 0)
    p["history"] = p["history"][:, :0]
    assert torch.equal(hs.adjust_logits(logits, **p), logits)


def test_many_rows(hs):
    """More rows than a launch has in one direction."""
    logits = torch.randn((65539, 5), device=DEV)
    history = torch.arange(65539, device=DEV, dtype=torch.int32)[:, None] % 5
    got = hs.adjust_logits(logits, history=history.contiguous(), presence=torch.ones(65539, device=DEV))
    want = logits.clone()
    want.scatter_add_(1, history.long(), torch.full((65539, 1), -1.0, device=DEV))
    assert torch.equal(got, want)


def test_rows_past_32_bits(hs):
    """The last row lies more than 2^32 bytes behind the first, in logits and out."""
    R, V = 17500, 128000
    logits = torch.zeros((R, V), dtype=torch.bfloat16, device=DEV)
    logits[-1] = 2.0
    history = torch.zeros((R, 1), dtype=torch.int32, device=DEV)
    history[-1] = V - 1
    got = hs.adjust_logits(logits, history=history, repetition=torch.full((R,), 2.0, device=DEV), out=logits)
    assert got[-1, -1] == 1.0 and (got[-1, :-1] == 2.0).all() and (got[:-1] == 0.0).all()


def test_long_history_counts(hs):
    """One word said a million times, before and after the prompt."""
    L = 1 << 20
    history = torch.full((2, L), 3, dtype=torch.int32, device=DEV)
    logits = torch.zeros((2, 4100), device=DEV)
    prompt = torch.tensor([0, L - 5], dtype=torch.int32, device=DEV)
    got = hs.adjust_logits(logits, history=history, prompt=prompt, frequency=torch.ones(2, device=DEV))
    assert got[0, 3] == -float(L) and got[1, 3] == -5.0 and got.count_nonzero() == 2


@pytest.mark.parametrize("dtype", BOTH)
def test_captured_and_replayed(hs, dtype):
    p = _rules(5, 3001, 200, 2, 2)
    logits = torch.randn((5, 3001), generator=_gen(0)).to(dtype).to(DEV)
    hs.adjust_logits(logits, **p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = hs.adjust_logits(logits, **p)
    for seed in range(4):
        new = _rules(5, 3001, 200, 2, 2, seed=seed + 9)
        for k, v in new.items():
            p[k].copy_(v)
        logits.copy_(torch.randn((5, 3001), generator=_gen(seed)))
        want = hs.adjust_logits(logits, **p)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_another_stream(hs):
    p = _rules(5, 3001, 200, 2, 2)
    logits = torch.randn((5, 3001), generator=_gen(0)).to(DEV)
    want = hs.adjust_logits(logits, **p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = hs.adjust_logits(logits, **p, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
