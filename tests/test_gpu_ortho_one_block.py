"""GPU: matrices that one block takes through all steps need no workspace: none is allocated, a capture needs no reservation
and a caller's workspace need not have room for them."""
import numpy as np
import pytest

from test_gpu_ortho import _dev, _sidco, _torch

pytestmark = pytest.mark.gpu

SHAPES = [(64, 576), (576, 64), (3, 5), (64, 129)]


def _case(rows, cols):
    torch = _torch()
    x = _dev(np.random.default_rng(rows).standard_normal((40, rows, cols)).astype(np.float32))
    want = torch.empty_like(x)
    _sidco().sidco_orthogonalize(x, want)
    torch.cuda.synchronize()
    return x, want, torch.empty_like(x)


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_nothing_is_allocated_and_a_first_call_can_be_captured(rows, cols):
    torch, sidco = _torch(), _sidco()
    x, want, out = _case(rows, cols)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out.zero_()  # what the runtime itself sets up for a stream's first kernel
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    sidco.sidco_orthogonalize(x, out, stream=s)
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free
    assert torch.equal(out, want)
    fresh = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=fresh):
        sidco.sidco_orthogonalize(x, out, stream=fresh)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_a_small_workspace_of_the_caller_is_enough(rows, cols):
    torch, sidco = _torch(), _sidco()
    x, want, out = _case(rows, cols)
    m, w = torch.zeros_like(x), torch.zeros_like(x)
    ws = torch.empty(sidco.sidco_workspace_bytes(1), dtype=torch.uint8, device="cuda")
    try:
        sidco.sidco_set_workspace(ws)
        sidco.sidco_orthogonalize(x, out)
        sidco.sidco_muon_step(x, m, w, lr=1.0, mu=0.0, scale=-1.0)
    finally:
        torch.cuda.synchronize()
        sidco.sidco_set_workspace(None)
    assert torch.equal(out, want)
    assert torch.equal(w, want)


def test_long_row_strides_take_the_other_way():
    """Row strides past 2^20 elements are served with a workspace."""
    torch, sidco = _torch(), _sidco()
    x, want, out = _case(6, 70)
    rows = torch.zeros((40, 6, (1 << 20) + 4), device="cuda")[:, :, 1:71]
    rows.copy_(x)
    sidco.sidco_orthogonalize(rows, out)
    assert float((out - want).norm()) <= 1e-4 * float(want.norm())
