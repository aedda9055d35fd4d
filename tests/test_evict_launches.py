"""An eviction's launches (CPU; see evict_launches.cpp)."""
import os
import re

from paper_2608_10402_amd.build import _hipcc
from test_staging_threads import CSRC, INC, ROOT, _run


def test_launches_of_any_number_of_tasks_and_heads(tmp_path):
    obj, exe = str(tmp_path / "evict.o"), str(tmp_path / "launches")
    _run([_hipcc(), "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", *INC, "-c",
          os.path.join(CSRC, "kv_evict.hip"), "-o", obj])
    fatbin = re.findall(r"\b__hip_fatbin\w*", _run(["nm", "-u", obj]))  # the device code that a full compile would embed
    _run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", *INC, os.path.join(ROOT, "tests", "evict_launches.cpp"),
          obj, *["-Wl,--defsym=%s=0" % s for s in fatbin], "-o", exe])
    assert _run([exe]).strip() == "ok"
