"""The plans of a layer of stored experts (CPU only; sizes alone)."""
import subprocess
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent


def test_plans_fit_their_workspace_and_all_pieces_add_alike(tmp_path):
    exe = tmp_path / "driver"
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Wno-unused-function", "-Wno-unused-variable",
                        "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                        str(ROOT / "paper_2608_28113_amd" / "csrc"), "-o", str(exe),
                        str(ROOT / "tests" / "native" / "expert_plan_driver.cpp")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "expert plans: ok" in r.stdout, r.stdout + r.stderr
