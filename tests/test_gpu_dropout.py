"""GPU: dropout from the counter-based generator against its definition."""
import math

import numpy as np
import pytest

import language_reference as ref

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _sidco():
    import paper_2101_10761_amd as sidco
    return sidco


def _dtype(t):
    torch = _torch()
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[t]


def _wide(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (1, 8), (5, 9), (3, 2049), (70, 150), (257, 64), (2, 20_000), (1000, 33)])
@pytest.mark.parametrize("t,o", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("p,add", [(0.5, False), (0.1, True), (0.0, False), (1.0, True), (1e-5, False)])
def test_dropout(rows, cols, t, o, p, add):
    torch, sidco = _torch(), _sidco()
    g = torch.Generator().manual_seed(rows * cols)
    gap = rows % 2 * 3
    x = torch.randn(rows, cols + gap, generator=g).to(_dtype(t)).to("cuda")[:, :cols]
    whole = torch.randn(rows, cols + gap, generator=g).to(_dtype(o)).to("cuda")
    residual = torch.randn(rows, cols + 2 * gap, generator=g).to(_dtype(o)).to("cuda")[:, :cols] if add else None
    before, y = whole.clone(), whole[:, :cols]
    seed, offset = 0xC0FFEE123456789A, 2**33 - 7
    sidco.sidco_dropout(x, y, p, seed, offset=offset, residual=residual)
    torch.cuda.synchronize()
    want = ref.dropout(_wide(x), p, seed, offset, _wide(residual) if add else None)
    alone = ref.dropout(_wide(x), p, seed, offset)
    info = torch.finfo(_dtype(o))
    # the scale, the product and the sum rounded to 32 bits, the result to its type
    bound = np.abs(alone) * 2.0**-23 * 1.01 + np.abs(want) * (2.0**-24 + info.eps / 2) * 1.01 + info.tiny * info.eps / 2
    got = _wide(y)
    assert (np.abs(got - want) <= bound).all()
    if not add:
        assert np.array_equal(got == 0, alone == 0)
    assert torch.equal(whole[:, cols:], before[:, cols:])


def test_backward_drops_what_the_forward_dropped():
    torch, sidco = _torch(), _sidco()
    x, dy = torch.randn(300, 77, device="cuda"), torch.randn(300, 77, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    sidco.sidco_dropout(x, y, 0.3, 5)
    sidco.sidco_dropout(dy, dx, 0.3, 5)
    assert torch.equal(y == 0, dx == 0)
    share = float((y == 0).double().mean())
    # 23100 draws: five standard deviations of their mean
    assert abs(share - 0.3) < 5 * math.sqrt(0.3 * 0.7 / 23100)


def test_in_place_and_dropped_infinities():
    torch, sidco = _torch(), _sidco()
    x = torch.full((64, 64), float("inf"), device="cuda")
    x[1::2] = float("nan")
    kept = torch.from_numpy(ref.numbers(64, 64, 9, 4) >= 32768).to("cuda")
    y = torch.empty_like(x)
    sidco.sidco_dropout(x, y, 0.5, 9, offset=4)
    assert bool((y[~kept] == 0).all()) and not bool(torch.isfinite(y[kept]).any())
    a = torch.randn(33, 50, device="cuda").half()
    r, want = torch.randn(33, 50, device="cuda").half(), torch.empty_like(a)
    sidco.sidco_dropout(a, want, 0.25, 1, residual=r)
    b, c = a.clone(), r.clone()
    sidco.sidco_dropout(b, b, 0.25, 1, residual=r)
    sidco.sidco_dropout(a, c, 0.25, 1, residual=c)
    assert torch.equal(b, want) and torch.equal(c, want)


def test_blocks_follow_each_other_and_strides_do_not_count():
    torch, sidco = _torch(), _sidco()
    x = torch.ones(40, 21, device="cuda")
    whole, half, wide = torch.empty_like(x), torch.empty_like(x), torch.empty(40, 60, device="cuda")
    sidco.sidco_dropout(x, whole, 0.4, 3)
    sidco.sidco_dropout(x[:15], half[:15], 0.4, 3)
    sidco.sidco_dropout(x[15:], half[15:], 0.4, 3, offset=sidco.sidco_dropout_blocks(15, 21))
    sidco.sidco_dropout(x, wide[:, 5:26], 0.4, 3)
    assert torch.equal(whole, half) and torch.equal(whole, wide[:, 5:26])
    other = torch.empty_like(x)
    sidco.sidco_dropout(x, other, 0.4, 4)
    assert not torch.equal(whole, other)


def test_captured_call_draws_others_as_its_counter_moves():
    torch, sidco = _torch(), _sidco()
    x, y = torch.randn(100, 64, device="cuda"), torch.empty(100, 64, device="cuda")
    moved = torch.zeros(1, dtype=torch.int64, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        sidco.sidco_dropout(x, y, 0.5, 77, offset=10, device_offset=moved, stream=s)
        moved.add_(sidco.sidco_dropout_blocks(100, 64))
    seen = []
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(y)
        sidco.sidco_dropout(x, want, 0.5, 77, offset=10 + 800 * i)
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        seen.append(y.clone())
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_far_elements():
    """Elements whose offsets pass 2^32."""
    torch, sidco = _torch(), _sidco()
    whole = torch.empty(3 * (2**31 - 1), dtype=torch.float16, device="cuda")
    x = whole.view(3, 2**31 - 1)  # the widest rows and row stride that a call takes
    x[:, -100:] = 1.0
    x[:, : -100] = 0.0
    sidco.sidco_dropout(x, x, 0.5, 8)
    per_row = 2**28
    for r in range(3):
        first = (2**31 - 101) // 8  # the block of the last hundred's first element
        n = ref.numbers(1, 8 * 14, 8, r * per_row + first)[0]
        at = (2**31 - 101) - 8 * first
        assert np.array_equal(_wide(x[r, -100:]), np.where(n[at:at + 100] >= 32768, 2.0, 0.0))
