"""The example that quantizes, serves and trains a layer through every
operator, at a small size."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

PATH = Path(__file__).resolve().parent.parent / "examples" / "serve_and_tune_adapters.py"


def test_the_loss_falls_and_single_tokens_answer_as_a_batch():
    spec = importlib.util.spec_from_file_location("serve_and_tune_adapters", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, together, alone, right = example.main(steps=30)
    torch.cuda.synchronize()
    first, last = sum(losses[:3]) / 3, sum(losses[-3:]) / 3
    assert last < 0.8 * first, losses
    # each is within 2^-8 of the exact value, and 2^-14 of the sum's terms
    bound = 2.0 ** -7 * together.double().abs() + 2.0 ** -9
    assert ((together.double() - alone.double()).abs() <= bound).all()
    assert right > 1.0 / 100
