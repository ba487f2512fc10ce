"""GPU: the embedding's lookup and its gradient against their definitions in 64 bits."""
import numpy as np
import pytest

import language_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["f32", "f16", "bf16"]


def _torch():
    import torch
    return torch


def _sidco():
    import paper_2101_10761_amd as sidco
    return sidco


def _dtype(t):
    torch = _torch()
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[t]


def _half_step(t):
    """A rounding to t is off by this at most, relative to the value, and by the second number near zero."""
    torch = _torch()
    info = torch.finfo(_dtype(t))
    return info.eps / 2, info.tiny * info.eps / 2


def _matrix(rows, cols, t, seed, gap=0, scale=1.0):
    """A matrix whose rows lie `gap` elements apart in a larger buffer that starts off their alignment, and the buffer."""
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    whole = (torch.randn(rows, cols + gap + (1 if gap else 0), generator=g) * scale).to(_dtype(t)).to("cuda")
    return (whole[:, 1:1 + cols] if gap else whole), whole


def _words(n, vocab, seed, wide, padding=0.0, hot=0.0):
    rng = np.random.default_rng(seed)
    w = np.floor(vocab ** rng.random(n)).astype(np.int64) - 1
    w = np.clip(w, 0, vocab - 1)
    w[rng.random(n) < hot] = vocab // 2
    w[rng.random(n) < padding] = rng.choice([-100, -1, vocab, vocab + 5])
    return w, _torch().from_numpy(w).to(_torch().int64 if wide else _torch().int32).to("cuda")


def _wide(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("n,dim,vocab", [(1, 1, 1), (1, 4096, 7), (3, 7, 100), (65, 8, 5), (700, 1500, 1000), (257, 513, 300), (5000, 64, 2000), (33, 9001, 11)])
@pytest.mark.parametrize("t,o", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "f16")])
def test_lookup(n, dim, vocab, t, o):
    torch, sidco = _torch(), _sidco()
    gap = n % 2 * 3
    table, _ = _matrix(vocab, dim, t, 1, gap)
    w, words = _words(n, vocab, 2, n % 3 == 0, padding=0.1)
    out, whole = _matrix(n, dim, o, 3, gap)
    before = whole.clone()
    sidco.sidco_embedding(table, words, out, scale=1.7)
    torch.cuda.synchronize()
    want = ref.embedding(_wide(table), w, float(np.float32(1.7)))
    rel, least = _half_step(o)
    # the product rounded to 32 bits, then to the result's type
    np.testing.assert_array_less(np.abs(_wide(out) - want), np.abs(want) * (rel + 2.0**-24 * 1.01) + least + 1e-300)
    if gap:
        assert torch.equal(whole[:, 0], before[:, 0]) and torch.equal(whole[:, 1 + dim:], before[:, 1 + dim:])


@pytest.mark.parametrize("n,dim,vocab,hot,padding", [
    (1, 1, 1, 0, 0), (1, 300, 50, 0, 0), (2, 8, 3, 0, 0), (63, 7, 5, 0, 0.2), (64, 513, 90, 0.5, 0), (700, 1500, 1000, 0, 0),
    (2048, 64, 70, 0, 0.1), (2049, 65, 4000, 0.9, 0), (5000, 520, 17, 0, 0), (4000, 33, 900, 1.0, 0), (300, 20, 40, 0, 1.0),
    (70_001, 24, 3000, 0.3, 0.1), (66_000, 8, 1, 0, 0)])
@pytest.mark.parametrize("t,o,accumulate", [("f32", "f32", False), ("bf16", "f32", True), ("f16", "f16", True), ("bf16", "bf16", False)])
def test_gradient(n, dim, vocab, hot, padding, t, o, accumulate):
    torch, sidco = _torch(), _sidco()
    gap = n % 2 * 5
    grad, _ = _matrix(n, dim, t, 4, gap)
    w, words = _words(n, vocab, 5, n % 3 == 0, padding, hot)
    grad[torch.from_numpy(~ref.inside(w, vocab)).to("cuda")] = float("nan")  # what stands in padding is not looked at
    table, whole = _matrix(vocab, dim, o, 6, gap)
    before = whole.clone()
    old = _wide(table)
    sidco.sidco_embedding_grad(grad, words, table, scale=0.75, accumulate=accumulate)
    torch.cuda.synchronize()
    want, size, count = ref.embedding_grad(_wide(grad), w, vocab, 0.75)
    got = _wide(table)
    rel, least = _half_step(o)
    # count additions, the scale (exact here) and the old value's addition, each rounded to 32 bits; the last to the result's
    bound = (count[:, None] + 2) * 2.0**-24 * size
    if accumulate:
        want = want + old
        bound = bound + 2.0**-24 * (np.abs(old) + size)
        assert np.array_equal(got[count == 0], old[count == 0])
    bound = bound + (np.abs(want) + bound) * rel + least
    bad = np.abs(got - want) > bound
    bad[count == 0] = got[count == 0] != want[count == 0]
    assert not bad.any(), (np.abs(got - want).max(), np.argwhere(bad)[:5])
    if gap:
        assert torch.equal(whole[:, 0], before[:, 0]) and torch.equal(whole[:, 1 + dim:], before[:, 1 + dim:])


def test_gradient_is_the_same_every_time():
    torch, sidco = _torch(), _sidco()
    w, words = _words(9000, 500, 7, True, 0.05, 0.2)
    grad, _ = _matrix(9000, 200, "f32", 8)
    outs = []
    for i in range(4):
        out = torch.empty(500, 200, device="cuda")
        sidco.sidco_embedding_grad(grad, words, out)
        # another call between, on the same workspace
        sidco.sidco_embedding_grad(grad[: 100 + 999 * i], words[: 100 + 999 * i], torch.empty(500, 200, device="cuda"))
        outs.append(out)
    torch.cuda.synchronize()
    assert all(torch.equal(o, outs[0]) for o in outs)


def test_gradient_of_infinities_stays_with_its_word():
    torch, sidco = _torch(), _sidco()
    w = np.array([3, 1, 3, 0, 2, 1])
    grad = torch.ones(6, 40, device="cuda")
    grad[2, 5], grad[4, 6], grad[1, 7], grad[5, 7] = float("inf"), float("nan"), float("inf"), float("-inf")
    out = torch.empty(5, 40, device="cuda")
    sidco.sidco_embedding_grad(grad, torch.from_numpy(w).to("cuda"), out)
    got = out.cpu().numpy()
    assert got[3, 5] == np.inf and np.isnan(got[2, 6]) and np.isnan(got[1, 7])
    got[3, 5], got[2, 6], got[1, 7] = 2, 1, 2
    assert np.array_equal(got, np.array([1, 2, 1, 2, 0])[:, None] * np.ones((5, 40)))


def test_gradient_against_differences():
    """The gradient of f(T) = sum of c * lookup(T) by central differences of f, which is linear: they differ by roundings only."""
    torch, sidco = _torch(), _sidco()
    vocab, dim, n = 9, 5, 30
    w, words = _words(n, vocab, 9, True, 0.1)
    table, c = torch.randn(vocab, dim, device="cuda"), torch.randn(n, dim, device="cuda")
    out, got = torch.empty(n, dim, device="cuda"), torch.empty(vocab, dim, device="cuda")

    def f(t):
        sidco.sidco_embedding(t, words, out, scale=2.0)
        return float((out.double() * c.double()).sum())

    sidco.sidco_embedding_grad(c, words, got, scale=2.0)
    size = ref.embedding_grad(_wide(c), w, vocab, 2.0)[1]
    for v in range(vocab):
        for k in range(dim):
            up, down = table.clone(), table.clone()
            up[v, k] += 1.0
            down[v, k] -= 1.0
            step = float(up[v, k].double() - down[v, k].double())
            # lookups times 2 are exact in 32 bits; the gradient's sum of up to n rows is rounded as often
            assert abs((f(up) - f(down)) / step - float(got[v, k])) <= (n + 2) * 2.0**-24 * size[v, k] + 1e-12


def test_captured_and_replayed_beside_eager_calls():
    torch, sidco = _torch(), _sidco()
    s = torch.cuda.Stream()
    n, dim, vocab = 3000, 96, 400
    _, words = _words(n, vocab, 10, True)
    words = words.clone()
    grad, out, table = torch.randn(n, dim, device="cuda"), torch.empty(vocab, dim, device="cuda"), torch.randn(vocab, dim, device="cuda")
    rows = torch.empty(n, dim, device="cuda")
    torch.cuda.synchronize()
    sidco.sidco_reserve(sidco.sidco_workspace_bytes_embedding_grad(n, dim), stream=s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        sidco.sidco_embedding(table, words, rows, scale=3.0, stream=s)
        sidco.sidco_embedding_grad(grad, words, out, scale=3.0, stream=s)
    for i in range(3):
        words.copy_(_words(n, vocab, 20 + i, True, 0.1 * i)[1])
        grad.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want_rows, want = torch.empty_like(rows), torch.empty_like(out)
        sidco.sidco_embedding(table, words, want_rows, scale=3.0)
        sidco.sidco_embedding_grad(grad, words, want, scale=3.0)
        torch.cuda.synchronize()
        assert torch.equal(rows, want_rows) and torch.equal(out, want)
    del graph
    sidco.sidco_release(stream=s)


def test_far_rows():
    """Rows whose offsets pass 2^31 and 2^32 elements."""
    torch, sidco = _torch(), _sidco()
    vocab, dim, ld = 1_200_000, 8, 4000
    whole = torch.empty(vocab * ld, dtype=torch.float16, device="cuda")
    table = whole.view(vocab, ld)[:, :dim]
    words = torch.tensor([0, 536_871, 1_073_742, vocab - 1, 1_073_741], device="cuda")
    table[words] = torch.arange(40, device="cuda").view(5, 8).half()
    out = torch.empty(5, 8, device="cuda")
    sidco.sidco_embedding(table, words, out)
    assert torch.equal(out, torch.arange(40, device="cuda").view(5, 8).float())
    sidco.sidco_embedding_grad(out, words, table, accumulate=True)
    assert torch.equal(table[words].float(), 2 * out)


@pytest.mark.parametrize("n", [3, 2049])
def test_gradient_of_a_table_of_more_rows_than_blocks_for_them(n):
    torch, sidco = _torch(), _sidco()
    vocab = 2**27 + 5
    words = torch.randint(0, vocab, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    words[:3] = torch.tensor([0, vocab - 1, vocab - 1], device="cuda")
    table = torch.full((vocab, 1), 3.0, dtype=torch.float16, device="cuda")
    sidco.sidco_embedding_grad(torch.ones(n, 1, device="cuda"), words, table)
    torch.cuda.synchronize()
    distinct, counts = torch.unique(words, return_counts=True)
    assert torch.equal(table[distinct, 0].long(), counts) and int((table != 0).sum()) == len(distinct)


def test_binding_refuses_other_shapes_and_types():
    torch, sidco = _torch(), _sidco()
    x, words = torch.zeros(6, 8, device="cuda"), torch.zeros(6, dtype=torch.int64, device="cuda")
    table, loss = torch.zeros(10, 8, device="cuda"), torch.zeros(6, device="cuda")
    for wrong in (lambda: sidco.sidco_embedding(table, words, x[:5]), lambda: sidco.sidco_embedding(table, words, x[:, :7]),
                  lambda: sidco.sidco_embedding_grad(x[:5], words, table), lambda: sidco.sidco_dropout(x, table, 0.5, 1),
                  lambda: sidco.sidco_dropout(x, x, 0.5, 1, residual=table), lambda: sidco.sidco_cross_entropy(x, table, words[:5], loss, None),
                  lambda: sidco.sidco_cross_entropy(x, table[:, :7], words, loss, None), lambda: sidco.sidco_cross_entropy(x, table, words, loss[:5], None),
                  lambda: sidco.sidco_cross_entropy_grad(x, table, words, loss, None, x_grad=table),
                  lambda: sidco.sidco_cross_entropy_grad(x, table, words, loss, None, weight_grad=x)):
        with pytest.raises(ValueError):
            wrong()
    for wrong in (lambda: sidco.sidco_embedding(table, words.float(), x), lambda: sidco.sidco_embedding(table, words[::2], x[:3]),
                  lambda: sidco.sidco_embedding(table.t(), words, x), lambda: sidco.sidco_embedding(table.double(), words, x),
                  lambda: sidco.sidco_embedding(table.cpu(), words, x), lambda: sidco.sidco_embedding(table, words.cpu(), x),
                  lambda: sidco.sidco_dropout(x, x, 0.5, 1, residual=x.half()), lambda: sidco.sidco_cross_entropy(x, table.half(), words, loss, None),
                  lambda: sidco.sidco_cross_entropy(x, table, words, loss.double(), None),
                  lambda: sidco.sidco_cross_entropy_grad(x, table, words, loss, None, x_grad=x.half())):
        with pytest.raises(TypeError):
            wrong()
    with pytest.raises(sidco.SidcoError):
        sidco.sidco_cross_entropy_grad(x, table, words, loss, None, weight_grad=table.half())
