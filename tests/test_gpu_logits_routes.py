"""Every kernel behind the rules on logits, with all rules, against 64 bits:
blocks of 2048, 4096 and 8192 words, histories of several rounds that end in
the middle of one."""
from __future__ import annotations

import pytest
import torch

from tests.test_gpu_logits import BOTH, DEV, _close, _gen, _rules, hs  # noqa: F401

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def _wanted(logits, p):
    """(float64 result, the sum of the absolute terms behind it), row by row."""
    l = logits.cpu().double()
    p = {k: v.cpu() for k, v in p.items()}
    R, V = l.shape
    L = p["history"].shape[1]
    size = l.abs()
    for r in range(R):
        n, first = (min(max(int(p[k][r]), 0), L) for k in ("length", "prompt"))
        words = p["history"][r, :n].long()
        real = (words >= 0) & (words < V)
        seen = torch.bincount(words[real], minlength=V) > 0
        count = torch.bincount(words[first:][real[first:]], minlength=V).double()
        rho, f, a = (float(p[k][r]) for k in ("repetition", "frequency", "presence"))
        l[r] = torch.where(seen, torch.where(l[r] > 0, l[r] / rho, l[r] * rho), l[r])
        size[r] += torch.where(seen, l[r].abs(), 0.0) + 2 * abs(f) * count + abs(a) * (count > 0)
        l[r] -= f * count + a * (count > 0)
        b, m = int(p["bias_row"][r]), int(p["mask_row"][r])
        if 0 <= b < p["bias"].shape[0]:
            l[r] += p["bias"][b].double()
            size[r] += p["bias"][b].double().abs()
        if 0 <= m < p["mask"].shape[0]:
            allowed = (p["mask"][m][:, None] >> torch.arange(32)) & 1
            l[r] = torch.where(allowed.flatten()[:V] > 0, l[r], float("-inf"))
    return l, size


CASES = [(2, 9001, 4001), (3, 20011, 4096), (65, 33001, 50), (64, 33003, 4095), (2, 20003, 16387), (1, 100003, 40001),
         (3, 8191, 4097), (65, 33001, 9001), (70, 33007, 16389), (300, 8195, 5003)]


@pytest.mark.parametrize("R,V,L", CASES)
@pytest.mark.parametrize("dtype", BOTH)
def test_every_kernel_with_all_rules(hs, R, V, L, dtype):  # noqa: F811
    logits = (torch.randn((R, V), generator=_gen(V)) * 3).to(dtype).to(DEV)
    p = _rules(R, V, L, 3, 4, seed=R + L)
    print(f"[rules {R} {V} {L}]", flush=True)
    got = hs.adjust_logits(logits, **p)
    _close(got, *_wanted(logits, p))
    assert torch.equal(hs.adjust_logits(logits, **p, out=logits), got)  # in place


@pytest.mark.parametrize("R,V,L", [(2, 20003, 16387), (65, 33001, 9001), (64, 33003, 4095)])
@pytest.mark.parametrize("dtype", BOTH)
def test_lengths_about_the_end_of_a_round(hs, R, V, L, dtype):  # noqa: F811
    """Histories that end, and prompts that do, just before, at and just after a
    round's end, a thread's four words' and the row's."""
    logits = (torch.randn((R, V), generator=_gen(L)) * 3).to(dtype).to(DEV)
    p = _rules(R, V, L, 1, 1, seed=L)
    ends = torch.tensor([v for e in (0, 4, 4096, 8192, 16384, L) for v in range(e - 2, e + 3)], dtype=torch.int32)
    ends = ends[ends <= L + 2]
    p["length"].copy_(ends[torch.randint(0, len(ends), (R,), generator=_gen(1))])
    p["prompt"].copy_(ends[torch.randint(0, len(ends), (R,), generator=_gen(2))])
    print(f"[ends {R} {V} {L}]", flush=True)
    _close(hs.adjust_logits(logits, **p), *_wanted(logits, p))
