"""GPU: a dense operator's call between the sparsifier's calls on a stream, one that needs more workspace than there is, leaves
what they keep there: the bad-index flag, the diagnostics, the controller's count, the fits and the addresses that a graph holds."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _sidco():
    import paper_2101_10761_amd as sidco
    return sidco


def _grad(seed, d):
    return _torch().from_numpy((np.random.default_rng(seed).standard_t(3.0, d) * 1e-3).astype(np.float32)).to("cuda")


def _outs(d, delta):
    torch, sidco = _torch(), _sidco()
    cap = sidco.sidco_out_capacity(d, delta)
    return (torch.zeros(cap, dtype=torch.int32, device="cuda"), torch.zeros(cap, device="cuda"),
            torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda"))


@pytest.fixture
def stream():
    s = _torch().cuda.Stream()
    yield s
    _torch().cuda.synchronize()
    _sidco().sidco_release(stream=s)


def _dense_call(s, side=1100):
    torch, sidco = _torch(), _sidco()
    x = torch.randn(side, side, device="cuda")
    y = torch.empty_like(x)
    torch.cuda.synchronize()
    sidco.sidco_orthogonalize(x, y, stream=s)
    torch.cuda.synchronize()
    return y


def _mx4_call(s):
    torch, sidco = _torch(), _sidco()
    rows, k, n = 3000, 9000, 64
    w = [torch.zeros(size(n, k), dtype=torch.uint8, device="cuda") for size in (sidco.sidco_mx4_code_bytes, sidco.sidco_mx4_scale_bytes)]
    x, y = torch.randn(rows, k, device="cuda"), torch.empty(rows, n, device="cuda")
    torch.cuda.synchronize()
    sidco.sidco_mx4_linear(x, *w, y, stream=s)
    torch.cuda.synchronize()


@pytest.mark.parametrize("call", [_dense_call, _mx4_call])
def test_bad_index_is_still_reported(stream, call):
    torch, sidco = _torch(), _sidco()
    dense = torch.zeros(1000, device="cuda")
    idx = torch.tensor([5, -1, 7], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    sidco.sidco_scatter_add(dense, idx, torch.ones(3, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda"), 1.0, stream=stream)
    call(stream)
    assert sidco.sidco_scatter_check(stream=stream)
    assert not sidco.sidco_scatter_check(stream=stream)


def test_diagnostics_and_fits_stay(stream):
    torch, sidco = _torch(), _sidco()
    d = 100_003
    g, outs = _grad(1, d), _outs(d, 0.01)
    torch.cuda.synchronize()
    sidco.sidco_compress(g, None, 0.01, sidco.DIST_EXP, 2, *outs, stream=stream)
    sidco.sidco_dgc(g, None, 0.01, 0.05, 3, *outs, stream=stream)
    sidco.sidco_fit(g, None, sidco.DIST_GPD, stream=stream)
    before = bytes(sidco.sidco_read_diag(stream=stream)), sidco.sidco_dgc_result(stream=stream), sidco.sidco_fit_result(stream=stream)
    _dense_call(stream)
    after = bytes(sidco.sidco_read_diag(stream=stream)), sidco.sidco_dgc_result(stream=stream), sidco.sidco_fit_result(stream=stream)
    assert before == after


def test_a_dense_call_alone_has_no_diagnostics(stream):
    sidco = _sidco()
    _dense_call(stream)
    assert not sidco.sidco_scatter_check(stream=stream)
    for read in (sidco.sidco_read_diag, sidco.sidco_fit_result, sidco.sidco_dgc_result):
        with pytest.raises(sidco.SidcoError):
            read(stream=stream)


def test_controller_keeps_its_window(stream):
    torch, sidco = _torch(), _sidco()
    d, Q = 200_003, 4
    out = []
    for between in (False, True):
        ctrl = sidco.Controller(0.001, sidco.DIST_EXP, stages=1, Q=Q)
        outs, seen = _outs(d, 0.001), []
        for i in range(2 * Q):
            g = _grad(20 + i, d)
            torch.cuda.synchronize()
            ctrl.compress(g, None, *outs, stream=stream)
            torch.cuda.synchronize()
            seen.append((ctrl.stages, int(outs[2]), ctrl.last_average))
            if between:
                _dense_call(stream, 300 + 200 * i)
        ctrl.close()
        out.append(seen)
    assert out[0] == out[1]


def test_repeated_calls_go_on(stream):
    """Calls that repeat a shape use what the one before left."""
    torch, sidco = _torch(), _sidco()
    d = 1_000_003
    g = _grad(5, d)
    want = None
    for between in (False, True):
        outs = _outs(d, 0.01)
        torch.cuda.synchronize()
        for i in range(3):
            sidco.sidco_compress(g, None, 0.01, sidco.DIST_EXP, 2, *outs, stream=stream)
            if between:
                _dense_call(stream, 500 + 300 * i)
            torch.cuda.synchronize()
        k = int(outs[2])
        got = k, set(outs[0][:k].tolist()), float(outs[3])
        want = want or got
        assert got[:2] == want[:2] and abs(got[2] - want[2]) <= 1e-5 * want[2]


def test_a_captured_sparsifier_call_outlives_a_larger_dense_call(stream):
    torch, sidco = _torch(), _sidco()
    d = 150_001
    g, outs, eager = _grad(7, d), _outs(d, 0.01), _outs(d, 0.01)
    sidco.sidco_reserve(sidco.sidco_workspace_bytes(d), stream=stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        sidco.sidco_compress(g, None, 0.01, sidco.DIST_EXP, 2, *outs, stream=stream)
    for i in range(3):
        _dense_call(stream, 600 + 500 * i)
        g.copy_(_grad(30 + i, d))
        graph.replay()
        torch.cuda.synchronize()
        sidco.sidco_compress(g, None, 0.01, sidco.DIST_EXP, 2, *eager)
        torch.cuda.synchronize()
        k = int(outs[2])
        assert k == int(eager[2]) and abs(float(outs[3]) - float(eager[3])) <= 1e-5 * float(eager[3])
        assert set(outs[0][:k].tolist()) == set(eager[0][:k].tolist())


def test_reserved_memory_serves_a_dense_call_and_release_frees_all():
    torch, sidco = _torch(), _sidco()
    s = torch.cuda.Stream()
    x = torch.randn(1500, 1500, device="cuda")
    y = torch.empty_like(x)
    need = sidco.sidco_workspace_bytes_orthogonalize(1, 1500, 1500, sidco.GRAD_F32)
    torch.cuda.synchronize()
    at_first = torch.cuda.mem_get_info()[0]
    sidco.sidco_reserve(need, stream=s)
    reserved = torch.cuda.mem_get_info()[0]
    assert at_first - reserved >= need
    sidco.sidco_orthogonalize(x, y, stream=s)
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == reserved
    sidco.sidco_release(stream=s)
    sidco.sidco_orthogonalize(x, y, stream=s)  # memory of its own
    torch.cuda.synchronize()
    sidco.sidco_release(stream=s)
    assert torch.cuda.mem_get_info()[0] >= at_first - (8 << 20)
