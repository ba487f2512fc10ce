"""CPU build of the host code of a language model's operators under -fsanitize=address,undefined, with a driver that calls their
host-only paths."""
import os
import re
import shutil

import pytest

from test_sanitizers import ENV, ROOT, SAN, _run

from paper_2101_10761_amd import build

LLVM = "/opt/rocm/llvm/bin/clang++"
SOURCES = ("sidco_embed.hip", "sidco_dropout.hip", "sidco_entropy.hip", "sidco_language_api.hip")


@pytest.mark.skipif(not os.path.exists(LLVM) or (shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc")),
                    reason="needs hipcc and its clang++")
def test_language_host_paths_under_address_and_undefined_sanitizers(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    objects, images = [], set()
    for source in SOURCES + ("driver",):
        path = os.path.join(SAN, "language_driver.cpp") if source == "driver" else os.path.join(build.CSRC, source)
        to = str(tmp_path / (source + ".o"))
        p = _run([hipcc, "-x", "hip", "--cuda-host-only", "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address",
                  "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-omit-frame-pointer", "-Wno-unused-command-line-argument", "-I",
                  os.path.join(ROOT, "include"), "-I", build.CSRC, "-c", path, "-o", to])
        assert p.returncode == 0, p.stderr
        objects.append(to)
        images.update(re.findall(r"__hip_fatbin_[0-9a-f]{1,16}", _run(["nm", to]).stdout))
    # no kernel is launched: the device images that these objects name are empty
    stub = tmp_path / "images.c"
    stub.write_text("".join(f"const char {name}[64];\n" for name in sorted(images)))
    exe = str(tmp_path / "language_san")
    p = _run([LLVM, "-g", "-O1", "-fsanitize=address,undefined", "-x", "c", str(stub), "-x", "none", *objects, "-L/opt/rocm/lib", "-lamdhip64",
              "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    assert p.returncode == 0, p.stderr
    r = _run([exe], env=ENV)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "0 failures" in r.stdout and "ERROR: AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stdout + r.stderr
