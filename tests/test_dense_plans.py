"""CPU: what the dense operators decide on the host, by the functions that they decide with (tests/host/plan_driver.hip)."""
import os
import shutil
import subprocess

import pytest

from paper_2101_10761_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plans") / "plans")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([HIPCC, *flags, "-w", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, os.path.join(HERE, "host", "plan_driver.hip"),
                    "-o", exe], check=True, capture_output=True)

    def run(questions):
        text = "".join(" ".join(str(v) for v in q) + "\n" for q in questions)
        out = subprocess.run([exe], input=text, check=True, capture_output=True, text=True).stdout.splitlines()
        assert len(out) == len(questions)
        return [[int(v) for v in line.split()] for line in out]

    return run


def test_stages_behind_the_last_have_no_offset(ask):
    """Every stage of every tile in order; the loads behind the last, of nothing, are of stage 0."""
    questions = [("sequence", stages, terms, tiles, blocks, block, depth)
                 for stages in (1, 2, 3, 5, 98) for terms in (1, 3) for tiles, blocks in ((1, 1), (7, 3), (513, 512), (256, 256))
                 for block in (0, blocks - 1) for depth in (2, 3, 4)]
    for q, (most,) in zip(questions, ask(questions)):
        assert most == 0, q
