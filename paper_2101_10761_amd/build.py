"""Builds libsidco.so (HIP, gfx950) in-tree.  Run as `python -m paper_2101_10761_amd.build`."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsidco.so")
SOURCES = ["sidco_kernels.hip", "sidco_topk.hip", "sidco_dgc.hip", "sidco_api.hip", "sidco_mx4.hip",
           "sidco_ortho.hip", "sidco_dense_api.hip", "sidco_embed.hip", "sidco_dropout.hip", "sidco_entropy.hip",
           "sidco_language_api.hip"]

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared",
    # packed fp32 VALU forms are kept out of the generated code on this target
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def build(verbose: bool = False) -> str:
    """Compiles every source, several at a time, and links the library."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        p = subprocess.run(cmd, capture_output=True, text=True)
        # hipcc's host pass warns that it does not know the packed-fp32 feature; that is expected
        err = "\n".join(l for l in p.stderr.splitlines() if "packed-fp32-ops" not in l)
        if p.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + err)
        if verbose and err.strip():
            print(err, file=sys.stderr)

    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        with ThreadPoolExecutor(4) as pool:
            list(pool.map(lambda so: run([hipcc, *flags, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(CSRC, so[0]), "-o", so[1]]),
                          zip(SOURCES, objects)))
        run([hipcc, *HIPCC_FLAGS, "-o", LIB, *objects])
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
