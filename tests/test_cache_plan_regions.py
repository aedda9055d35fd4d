"""Regions and order of the plans of the 4-bit attention and of eviction, checked by
tests/cache_plan_regions.cpp over random calls."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_10402_amd", "csrc")


def test_regions_and_order(tmp_path):
    exe = str(tmp_path / "cache_plan_regions")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    os.path.join(ROOT, "tests", "cache_plan_regions.cpp"), os.path.join(CSRC, "plan.cpp"), "-o", exe],
                   check=True, timeout=300)
    r = subprocess.run([exe, "400"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok 400", r.stdout + r.stderr[-2000:]
