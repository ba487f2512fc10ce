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


LARGE = {0: 256, 1: 192, 2: 128, 3: 64}


def test_products_of_the_tests_take_every_tile_and_both_ways(ask):
    """So that a change of the rules cannot take the tests away from a kernel unnoticed."""
    from test_gpu_mx4_tiles import PRODUCTS
    plans = ask([("plan", m, n, 1, -(-k // 256)) for m, n, k in PRODUCTS])
    whole = {pick for (m, n, k), (pick, columns, rest) in zip(PRODUCTS, plans) if columns == n}
    split = {(pick, rest) for (m, n, k), (pick, columns, rest) in zip(PRODUCTS, plans) if columns < n}
    assert whole == set(LARGE), plans
    assert {pick for pick, _ in split} == {0} and {rest for _, rest in split} == {1, 2, 3}, plans


def test_matrices_of_the_tests_take_every_tile_group_and_both_ways(ask):
    from test_gpu_ortho_tiles import COEF, SHAPES
    up = lambda v: -(-v // 64) * 64  # noqa: E731
    seen = {kind: {"symmetric": set(), "two": set(), "apply": set(), "split": set(), "group": set()} for kind in ("pairs", "halves")}
    for batch, rows, cols in SHAPES:
        for precision in ("halves", "bf16", "pairs"):
            paired = {"halves": 0, "bf16": -16, "pairs": -32}[precision]
            (one, paired, group, group_halves), = ask([("steps", batch, rows, cols, 5, paired, *COEF)])
            assert not one and paired == {"halves": 0, "bf16": 4, "pairs": 5}[precision]
            for kind, g, terms in (("pairs", group, 3), ("halves", group_halves, 1)):
                if g == 0:
                    continue
                s = seen[kind]
                lines = lambda c: up(c) * 2 // 128 * terms  # noqa: E731
                (gram,), (plain,), (two,), (pick, columns, rest) = ask([
                    ("triangle", rows, batch, lines(cols)), ("triangle", rows, batch, lines(rows)),
                    ("triangle", rows, 2 * batch, lines(rows)), ("plan", rows, cols, batch, lines(rows))])
                s["group"].add(g)
                s["symmetric"].add(plain)
                if g > 2:
                    s["two"].add(two)
                s["apply"].add(pick)
                if columns < cols:
                    s["split"].add((pick, rest))
    assert seen["pairs"]["group"] == {3, 4} and seen["halves"]["group"] == {1, 2}, seen
    for kind in seen:
        assert seen[kind]["symmetric"] >= {0, 2, 3} and 1 in seen["pairs"]["symmetric"], seen
        assert seen[kind]["apply"] >= {0, 1, 2}, seen
        assert {pick for pick, _ in seen[kind]["split"]} >= {0, 1} and len(seen[kind]["split"]) >= 3, seen
    assert seen["pairs"]["two"] >= {0, 1, 2, 3}, seen


def test_precision_and_groups_by_type(ask):
    coef = (3.4445, -4.7750, 2.0315)
    for steps, paired, coefs, want in (
            (5, -32, coef, 5), (5, -16, coef, 4), (1, -16, coef, 0), (100, -16, coef, 99),
            (5, -16, (4.5, -8.4, 3.5), 5),      # a step multiplies by more than 4
            (5, -16, (1.5, -0.5, 0.0), 4)):
        (one, got, group, halves), = ask([("steps", 4, 300, 5000, steps, paired, *coefs)])
        assert not one and got == want
        assert group <= (4 if got < steps else 3) and halves == (1 if got < steps else 0)
    for rows, cols, paired, one in ((64, 576, 5, 1), (577, 64, 5, 0), (64, 577, 0, 1), (768, 64, 0, 1), (64, 769, 0, 0), (65, 65, 5, 0), (1, 1, 5, 1)):
        assert ask([("steps", 1, rows, cols, 5, paired, *coef)])[0][0] == one
