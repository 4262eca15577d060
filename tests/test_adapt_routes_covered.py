"""Every way that the plans of the stored layer in use choose - kernel, tile,
split or whole - is taken by a test that compares it with 64 bits (CPU only:
the plans are asked, not run)."""
import math
import random
import subprocess

import pytest

from tests import test_gpu_adapt, test_gpu_adapt_plain, test_gpu_adapt_routes, test_gpu_adapt_tiles, test_gpu_loss
from tests import test_gpu_adapt_wide, test_gpu_loss_precision
from tests.test_adapt_plans import driver  # noqa: F401


def _sizes(test, names):
    """The values that a test is parametrized over."""
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0] == names)


def _tested():
    lines = []
    names = "T,n,m,count,rank,how"
    for case in (_sizes(test_gpu_adapt.test_linear_matches_64_bits, names)
                 + _sizes(test_gpu_adapt_routes.test_linear_on_both_sides_of_every_change, names)
                 + test_gpu_adapt_tiles.LINEAR + test_gpu_adapt_wide.LINEAR):
        lines.append("linear %d %d %d %d %d" % tuple(case[:5]))
    plain = test_gpu_adapt_plain.test_matches_64_bits_in_rows_of_any_stride
    lines += [f"linear {T} {n} {m} 0 0" for T in _sizes(plain, "T") for n, m in _sizes(plain, "n,m")]
    for case in (_sizes(test_gpu_adapt.test_gradients_match_64_bits, names)
                 + _sizes(test_gpu_adapt_routes.test_gradients_on_both_sides_of_every_change, names)
                 + test_gpu_adapt_tiles.GRAD):
        lines.append("grad %d %d %d %d %d" % tuple(case[:5]))
    for case in (test_gpu_loss.CASES + test_gpu_adapt_tiles.LOSS
                 + _sizes(test_gpu_adapt_routes.test_loss_of_few_tokens_and_words_of_many_k, "T,d,V")
                 + _sizes(test_gpu_loss_precision.test_gradients_are_rounded_to_bf16_once, "T,d,V")):
        lines += ["loss %d %d %d 0 0" % case, "loss_grad %d %d %d 0 0" % case]
    return lines + ["loss_grad 65600 16 10007 0 0"]  # test_gradient_over_several_pieces_of_the_vocabulary


def _calls(rng, count):
    """Calls over the whole range, each size spread over its logarithm."""
    def spread(most, by=1):
        return by * max(1, round(math.exp(rng.uniform(0.0, math.log(most / by)))))

    for _ in range(count):
        T, n, m, adapters, rank = spread(16384), spread(16384, 16), spread(16384), spread(64), spread(256, 8)
        yield f"linear {T} {n} {m} {adapters} {rank}"
        yield f"linear {T} {n} {m} 0 0"
        yield f"grad {T} {n} {m} {adapters} {rank}"
        T, d, vocab = spread(16384), spread(8192, 16), spread(160000)
        yield f"loss {T} {d} {vocab} 0 0"
        yield f"loss_grad {T} {d} {vocab} 0 0"


def _ways(exe, lines):
    r = subprocess.run([str(exe), "ways"], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    taken = {}
    for line, ways in zip(lines, r.stdout.splitlines(), strict=False):
        for way in ways.split():
            taken.setdefault(way, line)
    assert len(r.stdout.splitlines()) == len(lines)
    return taken


@pytest.mark.parametrize("seed", [0, 1])
def test_every_way_that_a_plan_chooses_is_tested(driver, seed):  # noqa: F811
    tested = _ways(driver, _tested())
    chosen = _ways(driver, list(_calls(random.Random(seed), 20000)))
    missing = {way: line for way, line in chosen.items() if way not in tested}
    assert not missing, missing
    assert len(chosen) > 80
