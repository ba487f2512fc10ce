"""CPU build of the whole library's host code under -fsanitize=address,undefined with a driver that calls the dense operators'
host-only paths."""
import os
import shutil
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_sanitizers import ENV, ROOT, SAN, _run

from paper_2101_10761_amd import build

LLVM = "/opt/rocm/llvm/bin/clang++"


@pytest.mark.skipif(not os.path.exists(LLVM) or (shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc")),
                    reason="needs hipcc and its clang++")
def test_dense_host_paths_under_address_and_undefined_sanitizers(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    exe = str(tmp_path / "dense_san")
    objects = [str(tmp_path / (s + ".o")) for s in build.SOURCES]

    def compile_one(source, to):
        return _run([hipcc, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                     "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-omit-frame-pointer",
                     "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "-c",
                     os.path.join(build.CSRC, source), "-o", to])

    with ThreadPoolExecutor(4) as pool:
        for p in pool.map(compile_one, build.SOURCES, objects):
            assert p.returncode == 0, "\n".join(l for l in p.stderr.splitlines() if "packed-fp32-ops" not in l)
    p = _run([LLVM, "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined", "-I", os.path.join(ROOT, "include"),
              os.path.join(SAN, "dense_driver.cpp"), *objects, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    assert p.returncode == 0, p.stderr
    r = _run([exe], env=ENV)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "0 failures" in r.stdout and "ERROR: AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stdout + r.stderr
