"""The tile products' matrix instructions are written out, and with them the waits around the sums they add to (see
sidco_product.h): this reads the AMD assembly that the compiler makes of the sources here and checks that it leaves the sums
alone between the first product and the wait after the last one, and reads and writes no scratch memory there."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2101_10761_amd import build

SOURCES = ("sidco_mx4.hip", "sidco_ortho.hip")


def _assembly(source, to):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    subprocess.run([hipcc, *flags, "-w", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-S", "--cuda-device-only",
                    os.path.join(build.CSRC, source), "-o", to], check=True, capture_output=True)
    return open(to).read()


def _kernels(text):
    return re.findall(r"^(_ZN5sidco\S*):.*?\n(.*?)s_endpgm", text, re.S | re.M)


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
def test_sums_are_left_alone_between_products(tmp_path):
    with ThreadPoolExecutor(2) as pool:
        texts = list(pool.map(_assembly, SOURCES, [str(tmp_path / (s + ".s")) for s in SOURCES]))
    seen = 0
    for text in texts:
        for name, body in _kernels(text):
            lines = [line.split(";")[0].strip() for line in body.split("\n")]
            if not any(line.startswith("buffer_load_dwordx4") and line.endswith("lds") for line in lines):
                continue  # not a tile product
            seen += 1
            products = [i for i, line in enumerate(lines) if line.startswith("v_mfma")]
            waits = [i for i, line in enumerate(lines) if line == "s_nop 15"]
            assert products and waits, name
            for first, last in [(products[0], max(products))]:
                end = min(i for i in waits if i > last)
                for line in lines[first:end]:
                    assert "accvgpr" not in line and "scratch_" not in line, (name, line)
                    if line.startswith("v_mfma"):
                        # the sum is added to in place
                        regs = re.findall(r"a\[\d+:\d+\]", line)
                        assert len(regs) == 2 and regs[0] == regs[1], (name, line)
                    else:
                        assert not re.search(r"\ba\[?\d", line), (name, line)
            # each half's products start behind a wait for what may have written their operands
            assert sum(line == "s_nop 3" for line in lines) >= 2, name
    assert seen >= 40
