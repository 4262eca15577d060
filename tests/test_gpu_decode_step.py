"""Routing, stored experts, a stored head and the rules on logits together, as
a decode step uses them."""
from __future__ import annotations

import sys
from pathlib import Path

import pytest
import torch

from tests import adapt_ref, decode_ref

sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.fixture(scope="module")
def served():
    import serve_experts
    yield serve_experts.main(steps=12)
    torch.cuda.empty_cache()


def test_the_rules_hold(served):
    _, rules, answers, _ = served
    assert answers.shape == (5, 12) and (answers >= 0).all()
    assert (answers[-1] % 2 == 0).all() and not (answers[0] == 7).any()
    # With these penalties no word comes twice in a row.
    assert (answers[:, 1:] != answers[:, :-1]).all()
    assert torch.equal(rules["history"][:, 4:].cpu(), answers)


def test_each_step_is_what_64_bits_say(served):
    """Every replayed step's choice against the whole step in 64 bits: its word's
    logit there is the largest, up to what the step's roundings are worth: bf16
    hidden states and logits, each half a step of 8 bits, on sums of terms."""
    import paper_2608_28113_amd as hs
    model, rules, answers, (history, length, token) = served
    head = adapt_ref.weights(model.head_scale, *model.head)
    history, length, token = history.cpu().clone(), length.cpu().clone(), token.cpu().clone()
    fixed = {k: v.cpu() for k, v in rules.items() if k not in ("history", "length")}
    for i in range(answers.shape[1]):
        X = model.embedding[token.to(model.embedding.device)]
        routed = X @ model.router.t()
        expert, weight = decode_ref.route(routed, model.k, True)
        got = hs.route_tokens(routed, model.k)
        assert torch.equal(got[0].cpu(), expert)
        Y, off = decode_ref.experts(X, expert, weight, *model.experts, sums=2.0 ** -14)
        Y = X.cpu().double() + Y
        off = off + 2.0 ** -8 * Y.abs()  # the sum with X, rounded too
        l = Y @ head.t()
        worth = off @ head.abs().t() + 2.0 ** -8 * l.abs() + 2.0 ** -14 * (Y.abs() @ head.abs().t())
        want, size = decode_ref.logits(l, history=history, length=length, **fixed)
        worth = 1.3 * worth + 2.0 ** -8 * want.abs().nan_to_num(posinf=0.0, neginf=0.0) + 2.0 ** -21 * size
        chosen = answers[:, i].long()
        at = want.gather(1, chosen[:, None])
        assert at.isfinite().all()
        slack = worth.max(-1, keepdim=True).values + worth.gather(1, chosen[:, None])
        assert (at + slack >= want.max(-1, keepdim=True).values).all(), i
        history.scatter_(1, length[:, None].long(), chosen[:, None].int())
        length += 1
        token = chosen


def test_tokens_alone_and_together(served):
    """A token's logits, alone and among others: equal up to the roundings of the
    hidden states to bf16, where a sum in another order tips one."""
    model = served[0]
    token = torch.arange(40, device=model.embedding.device) * 7
    together = model.logits(token)
    alone = torch.cat([model.logits(token[t:t + 1]) for t in range(40)])
    scale = together.float().abs().max()
    assert ((together.float() - alone.float()).abs() <= 2.0 ** -5 * scale).all()
