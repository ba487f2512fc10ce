"""CPU: no call of a language model's operators asks for more workspace than the library says that one of its sizes needs, however
its operands lie.  The library's host code is built with a driver that stands in for the workspace and notes what it is asked for."""
import os
import re
import shutil

import pytest

from test_sanitizers import ROOT, SAN, _run
from test_sanitizers_language import LLVM, SOURCES

from paper_2101_10761_amd import build


@pytest.mark.skipif(not os.path.exists(LLVM) or (shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc")),
                    reason="needs hipcc and its clang++")
def test_calls_ask_for_what_the_library_says_at_most(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    objects, images = [], set()
    for source in SOURCES + ("driver",):
        path = os.path.join(SAN, "workspace_driver.cpp") if source == "driver" else os.path.join(build.CSRC, source)
        to = str(tmp_path / (source + ".o"))
        p = _run([hipcc, "-x", "hip", "--cuda-host-only", "-O1", "-std=c++17", "--offload-arch=gfx950", "-I", os.path.join(ROOT, "include"), "-I",
                  build.CSRC, "-c", path, "-o", to])
        assert p.returncode == 0, p.stderr
        objects.append(to)
        images.update(re.findall(r"__hip_fatbin_[0-9a-f]{1,16}", _run(["nm", to]).stdout))
    # no kernel is launched: the device images that these objects name are empty
    stub = tmp_path / "images.c"
    stub.write_text("".join(f"const char {name}[64];\n" for name in sorted(images)))
    exe = str(tmp_path / "workspace")
    p = _run([LLVM, "-O1", "-x", "c", str(stub), "-x", "none", *objects, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    assert p.returncode == 0, p.stderr
    r = _run([exe])
    assert r.returncode == 0 and " 0 failures" in r.stdout, r.stdout[-3000:] + r.stderr
