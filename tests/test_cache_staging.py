"""Launches that report an error while a kernel that reads a staging slot is queued (CPU; see
cache_staging.cpp)."""
import os
import re

from paper_2608_10402_amd.build import _hipcc
from test_staging_threads import CSRC, INC, ROOT, _run


def test_a_queued_reader_keeps_its_plan_when_the_call_fails(tmp_path):
    objs = [str(tmp_path / (src + ".o")) for src in ("tide_api", "cache_api")]
    for obj in objs:
        src = os.path.join(CSRC, os.path.basename(obj)[:-2] + ".hip")
        _run([_hipcc(), "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", *INC, "-c", src,
              "-o", obj])
    # the device code that a full compile would embed
    fatbin = set(re.findall(r"\b__hip_fatbin\w*", "".join(_run(["nm", "-u", obj]) for obj in objs)))
    exe = str(tmp_path / "staging")
    _run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", *INC, os.path.join(ROOT, "tests", "cache_staging.cpp"),
          os.path.join(CSRC, "plan.cpp"), *objs, *["-Wl,--defsym=%s=0" % s for s in sorted(fatbin)], "-o", exe,
          "-pthread"])
    assert _run([exe]).strip() == "ok"
