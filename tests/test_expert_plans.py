"""The plans of a layer of stored experts (CPU only; sizes alone)."""
import math
import random
import subprocess
from pathlib import Path

import pytest

from tests import test_gpu_experts_exact, test_gpu_experts_pieces

ROOT = Path(__file__).resolve().parent.parent


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    """The plans alone, built from expert_plan.h."""
    exe = tmp_path_factory.mktemp("plan") / "driver"
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Wno-unused-function", "-Wno-unused-variable",
                        "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                        str(ROOT / "paper_2608_28113_amd" / "csrc"), "-o", str(exe),
                        str(ROOT / "tests" / "native" / "expert_plan_driver.cpp")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return exe


def test_plans_fit_their_workspace_and_all_pieces_add_alike(driver):
    r = subprocess.run([str(driver)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "expert plans: ok" in r.stdout, r.stdout + r.stderr


def _ways(driver, calls):
    lines = "".join("%d %d %d %d %d\n" % c for c in calls)
    r = subprocess.run([str(driver), "ways"], input=lines, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    return {way: call for call, line in zip(calls, r.stdout.splitlines(), strict=False) for way in line.split()}


def test_every_way_is_compared_with_one_right_value(driver):
    """What the plans choose over the whole range of sizes is among what the tests
    on exact numbers take, and every number of waves among calls in pieces."""
    rng = random.Random(7)

    def spread(most, by=1):
        return by * max(1, round(math.exp(rng.uniform(0.0, math.log(most / by)))))

    calls = [(spread(16384), spread(16384, 16), spread(16384, 16), (e := spread(512)), spread(min(e, 32)))
             for _ in range(40000)]
    exact = _ways(driver, test_gpu_experts_exact.SMALL + test_gpu_experts_exact.WIDE)
    missing = {way: call for way, call in _ways(driver, calls).items() if way not in exact}
    assert not missing, missing
    pieces = _ways(driver, test_gpu_experts_pieces.CALLS)
    assert {w.split(":")[2] for w in pieces if w.startswith("gate")} == {"1", "2", "4"}, pieces
