"""Host code of the adapted layer and the token loss under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only; GPU code is compiled normally and never
launched)."""
import os
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not Path(HIPCC).exists(), reason="hipcc not installed")
def test_plans_and_validation_are_sanitizer_clean(tmp_path):
    csrc = ROOT / "paper_2608_28113_amd" / "csrc"
    common = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-ffp-contract=off",
              "-fhip-fp32-correctly-rounded-divide-sqrt", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
              "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
              "-Xarch_host", "-fno-omit-frame-pointer", "-I", str(ROOT / "include"), "-I", str(csrc)]
    units = [(csrc / f"{u}.hip", tmp_path / f"{u}.o") for u in ("adapt", "loss")]
    units.append((ROOT / "tests" / "native" / "adapt_sanitize_driver.cpp", tmp_path / "driver.o"))
    exe = tmp_path / "driver"
    for src, obj in units:
        r = subprocess.run(common + ["-x", "hip", "-c", "-o", str(obj), str(src)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address",
                        "-Xarch_host", "-fsanitize=undefined", "-o", str(exe), *[str(o) for _, o in units], "-lm"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "sanitize driver: ok" in r.stdout, (r.stdout + r.stderr)[-3000:]
