"""GPU: a workspace of the size that the library says is enough for a language model's operators, for calls of few rows too."""
import pytest

from test_gpu_cross_entropy import _case, _run, _sidco, _torch

pytestmark = pytest.mark.gpu

# 16-bit weights between whole lines, which the kernel for few rows takes up to 96 of, and the same out of its reach
SIZES = [(96, 100, 1000, "bf16", 0), (64, 72, 700, "f16", 0), (33, 500, 50, "bf16", 0), (96, 66, 300, "bf16", 1), (33, 8, 10, "f16", 0), (40, 101, 90, "f16", 0),
         (32, 64, 20, "bf16", 0), (80, 40, 120, "f32", 0)]


@pytest.mark.parametrize("n,dim,vocab,t,gap", SIZES)
def test_a_callers_workspace(n, dim, vocab, t, gap):
    torch, sidco = _torch(), _sidco()
    x, w, words = _case(n, dim, vocab, t, gap=gap)
    want = _run(x, w, words)
    code = {"f32": sidco.GRAD_F32, "f16": sidco.GRAD_F16, "bf16": sidco.GRAD_BF16}[t]
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    space = torch.empty(sidco.sidco_workspace_bytes_cross_entropy(n, dim, vocab, code), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    sidco.sidco_set_workspace(space)  # a call that needs more is refused
    try:
        sidco.sidco_cross_entropy(x, w, words, loss, lse)
        torch.cuda.synchronize()
    finally:
        sidco.sidco_set_workspace(None)
    assert torch.equal(loss, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("n,dim,vocab,t,gap", SIZES[:3])
def test_a_captured_call_keeps_to_what_was_reserved(n, dim, vocab, t, gap):
    """A larger call on the stream between replays, which has memory of its own, does not touch the graph's."""
    torch, sidco = _torch(), _sidco()
    x, w, words = _case(n, dim, vocab, t, gap=gap)
    want = _run(x, w, words)
    code = {"f16": sidco.GRAD_F16, "bf16": sidco.GRAD_BF16}[t]
    s = torch.cuda.Stream()
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    large = _case(700, 100, 3000, "f32")
    out = torch.empty(700, device="cuda")
    torch.cuda.synchronize()
    sidco.sidco_reserve(sidco.sidco_workspace_bytes_cross_entropy(n, dim, vocab, code), stream=s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        sidco.sidco_cross_entropy(x, w, words, loss, lse, stream=s)
    for i in range(3):
        with torch.cuda.stream(s):
            sidco.sidco_cross_entropy(*large, out, None)
        torch.cuda.synchronize()
        loss.fill_(-1.0), lse.fill_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(lse, want[1])
    del graph
    sidco.sidco_release(stream=s)
