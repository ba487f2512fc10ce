"""The cross entropy's products are the tile products' (see sidco_product.h), with other code around them: as for those, the AMD
assembly that the compiler makes of the source here leaves the sums alone between the first product and the wait after the last
one, and reads and writes no scratch memory there."""
import os
import re
import shutil

import pytest

from test_generated_code import _assembly, _kernels


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
def test_sums_are_left_alone_between_products(tmp_path):
    seen = 0
    for name, body in _kernels(_assembly("sidco_entropy.hip", str(tmp_path / "entropy.s"))):
        lines = [line.split(";")[0].strip() for line in body.split("\n")]
        if not any(line.startswith("buffer_load_dwordx4") and line.endswith("lds") for line in lines):
            continue
        seen += 1
        products = [i for i, line in enumerate(lines) if line.startswith("v_mfma")]
        last = max(products)
        end = min(i for i, line in enumerate(lines) if line == "s_nop 15" and i > last)
        for line in lines[products[0]:end]:
            assert "accvgpr" not in line and "scratch_" not in line, (name, line)
            if line.startswith("v_mfma"):
                regs = re.findall(r"a\[\d+:\d+\]", line)
                assert len(regs) == 2 and regs[0] == regs[1], (name, line)
            else:
                assert not re.search(r"\ba\[?\d", line), (name, line)
        assert sum(line == "s_nop 3" for line in lines) >= 2, name
    assert seen >= 40
