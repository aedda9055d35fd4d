"""The plans of the 4-bit cache, attention mass and eviction, checked by tests/cache_plan_check.cpp
over random calls, once plainly and once under host sanitizers."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_10402_amd", "csrc")


@pytest.mark.parametrize("flags,calls", [(["-O2"], 400), (["-O1", "-g", "-fsanitize=address,undefined",
                                                          "-fno-sanitize-recover=all"], 60)])
def test_cache_plans(tmp_path, flags, calls):
    exe = str(tmp_path / "cache_plan_check")
    subprocess.run(["g++", "-std=c++17", *flags, "-Wall", "-Wextra", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    os.path.join(ROOT, "tests", "cache_plan_check.cpp"), os.path.join(CSRC, "plan.cpp"), "-o", exe],
                   check=True, timeout=300)
    r = subprocess.run([exe, str(calls)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok %d" % calls, r.stdout + r.stderr[-2000:]
