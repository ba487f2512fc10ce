"""GPU: a language model's operators on parts of larger matrices, read where they are: what stands beside and behind them is no number, is not
looked at and is left as it was."""
import pytest

from test_gpu_cross_entropy import _case, _dtype, _run, _sidco, _torch

pytestmark = pytest.mark.gpu


def _within(t, before, after, behind):
    """A view with t's values in a matrix of NaN with that many more columns before and after and rows behind, and the matrix."""
    torch = _torch()
    whole = torch.full((t.shape[0] + behind, before + t.shape[1] + after), float("nan"), dtype=t.dtype, device="cuda")
    view = whole[:t.shape[0], before:before + t.shape[1]]
    view.copy_(t)
    return view, whole


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,dim,vocab", [(3, 64, 700), (33, 128, 500), (150, 64, 1000), (300, 192, 2050), (90, 72, 300)])
@pytest.mark.parametrize("before,after", [(0, 64), (8, 56), (64, 128), (3, 2)])
def test_cross_entropy(t, n, dim, vocab, before, after):
    torch, sidco = _torch(), _sidco()
    x, w, words = _case(n, dim, vocab, t)
    x, w = x.contiguous(), w.contiguous()
    g = torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    want = _run(x, w, words, g)
    vx, wx = _within(x, before, after, 200)
    vw, ww = _within(w, before, after, 300)
    got = _run(vx, vw, words, g)
    # fp32 rows are multiplied alike wherever they start; of 16-bit ones few rows are by a kernel of their own if they start at whole words
    if t == "f32" or n <= 32 or n > 96:
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    else:
        for a, b in zip(got, want):
            # sums of up to 128 products in another order, (128 + 16) 2^-24 = 9e-6, and roundings to 16 bits that fall to the other side
            assert float((a.double() - b.double()).norm()) <= (1e-5 if a.dtype is torch.float32 else 2.0**-7) * float(b.double().norm())
    dx, wdx = _within(torch.zeros_like(x), before, after, 5)
    dw, wdw = _within(torch.zeros_like(w), before, after, 5)
    loss, lse = want[0], want[1]
    sidco.sidco_cross_entropy_grad(vx, vw, words, lse, g, dx, dw, accumulate=True, loss=loss)
    torch.cuda.synchronize()
    ax, aw = torch.empty_like(x), torch.zeros_like(w)
    sidco.sidco_cross_entropy_grad(x, w, words, lse, g, ax, aw, accumulate=True, loss=loss)
    torch.cuda.synchronize()
    assert torch.equal(dx, ax) and torch.equal(dw, aw)
    for view, whole in ((vx, wx), (vw, ww), (dx, wdx), (dw, wdw)):
        assert int(torch.isnan(whole).sum()) == whole.numel() - view.numel()


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,dim", [(5, 9), (700, 1111), (2049, 520), (8300, 7)])
def test_embedding_and_dropout(t, n, dim):
    torch, sidco = _torch(), _sidco()
    vocab = 901
    gen = torch.Generator(device="cuda").manual_seed(n)
    table, grad = (torch.randn(r, dim, device="cuda", generator=gen).to(_dtype(t)) for r in (vocab, n))
    words = torch.randint(-3, vocab + 3, (n,), device="cuda", generator=gen)
    vt, _ = _within(table, 3, 2, 9)
    vg, _ = _within(grad, 1, 0, 9)
    for accumulate in (False, True):
        a, b = table.clone(), _within(table, 5, 4, 3)
        sidco.sidco_embedding_grad(grad, words, a, scale=0.5, accumulate=accumulate)
        sidco.sidco_embedding_grad(vg, words, b[0], scale=0.5, accumulate=accumulate)
        assert torch.equal(a, b[0]) and int(torch.isnan(b[1]).sum()) == b[1].numel() - a.numel()
    a, b = torch.empty_like(grad), _within(grad, 5, 4, 3)
    sidco.sidco_embedding(table, words, a, scale=3.0)
    sidco.sidco_embedding(vt, words, b[0], scale=3.0)
    assert torch.equal(a, b[0]) and int(torch.isnan(b[1]).sum()) == b[1].numel() - a.numel()
    r, _ = _within(grad, 7, 1, 1)
    sidco.sidco_dropout(grad, a, 0.3, 4, residual=grad)
    sidco.sidco_dropout(vg, b[0], 0.3, 4, residual=r)
    assert torch.equal(a, b[0]) and int(torch.isnan(b[1]).sum()) == b[1].numel() - a.numel()


def test_captured_calls_of_few_words_and_rows():
    """Calls of one launch and their successors, replayed with other words, beside eager ones on another stream."""
    torch, sidco = _torch(), _sidco()
    n, dim, vocab = 60, 100, 400
    x, w, words = _case(n, dim, vocab, "f16")
    x, w, words = x.contiguous(), w.contiguous(), words.clone()
    s = torch.cuda.Stream()
    loss, lse, g = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.ones(n, device="cuda")
    dx, table, rows = torch.empty_like(x), torch.empty(vocab, dim, device="cuda"), torch.empty_like(x)
    torch.cuda.synchronize()
    need = [sidco.sidco_workspace_bytes_cross_entropy(n, dim, vocab, sidco.GRAD_F16), sidco.sidco_workspace_bytes_embedding_grad(n, dim),
            sidco.sidco_workspace_bytes_cross_entropy_grad(n, dim, vocab, sidco.GRAD_F16, sidco.GRAD_F32)]
    sidco.sidco_reserve(max(need), stream=s)

    def step(stream, rows, loss, lse, dx, table):
        sidco.sidco_embedding(w, words, rows, stream=stream)
        sidco.sidco_cross_entropy(x, w, words, loss, lse, stream=stream)
        sidco.sidco_cross_entropy_grad(x, w, words, lse, g, dx, table, stream=stream, loss=loss)
        sidco.sidco_embedding_grad(dx, words, table, accumulate=True, stream=stream)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(s, rows, loss, lse, dx, table)
    for i in range(4):
        a, b, c = _case(n, dim, vocab, "f16", seed=i, padding=0.3 * i)
        x.copy_(a), w.copy_(b), words.copy_(c), g.uniform_().mul_(2.0 ** (-12 * i))
        g[0] = 1.0
        torch.cuda.synchronize()
        graph.replay()
        want = [torch.empty_like(o) for o in (rows, loss, lse, dx, table)]
        step(None, *want)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((rows, loss, lse, dx, table), want))
    del graph
    sidco.sidco_release(stream=s)
