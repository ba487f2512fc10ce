"""GPU: lookups whose threads have four rows under way, the table's gradient around each of the sort's rules, and dropout of more
rows than blocks, against their definitions in 64 bits."""
import numpy as np
import pytest

import language_reference as ref
from test_gpu_embedding import _dtype, _half_step, _matrix, _sidco, _torch, _words

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,dim,gap", [(8192, 2049, 0), (8195, 2049, 3), (8197, 1032, 0), (262_147, 64, 3), (2_097_157, 5, 1), (16_385, 700, 0)])
@pytest.mark.parametrize("t,o", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
def test_long_lookups(n, dim, gap, t, o):
    torch, sidco = _torch(), _sidco()
    vocab = 3001
    table, _ = _matrix(vocab, dim, t, 1, gap)
    w, words = _words(n, vocab, 2, n % 2 == 0, padding=0.1)
    whole = torch.full((n, dim + gap), 5.0, dtype=_dtype(o), device="cuda")
    out = whole[:, gap:]
    sidco.sidco_embedding(table, words, out, scale=1.7)
    torch.cuda.synchronize()
    inside = torch.from_numpy(ref.inside(w, vocab)).to("cuda")
    want = torch.where(inside[:, None], table.double()[torch.where(inside, words.long(), 0)] * float(np.float32(1.7)), 0.0)
    rel, least = _half_step(o)
    # the product rounded to 32 bits, then to the result's type
    assert bool(((out.double() - want).abs() <= want.abs() * (rel + 2.0**-24 * 1.01) + least).all())
    assert bool((whole[:, :gap] == 5.0).all())


def test_a_lookup_of_more_rows_than_blocks_take_at_once():
    torch, sidco = _torch(), _sidco()
    n, dim, vocab = 4 * 2**20 + 7, 1025, 300
    table = torch.randn(vocab, dim, device="cuda").half()
    words = torch.randint(-1, vocab, (n,), device="cuda")
    out = torch.empty(n, dim, dtype=torch.float16, device="cuda")
    sidco.sidco_embedding(table, words, out, scale=2.0)
    doubled = torch.cat([table * 2, torch.zeros(1, dim, dtype=torch.float16, device="cuda")])
    for r in range(0, n, 2**18):
        assert torch.equal(out[r:r + 2**18], doubled[words[r:r + 2**18]]), r


@pytest.mark.parametrize("n,dim,vocab,hot,padding", [
    (2049, 5, 600, 0, 0.1), (8192, 1111, 900, 0.2, 0), (8193, 1111, 5000, 0, 0.1), (9001, 1111, 3000, 0.3, 0), (9001, 7, 40, 0, 0.1), (20_000, 200, 70_000, 0, 0.05),
    (65_536, 519, 20_000, 0, 0), (65_537, 519, 20_000, 0.1, 0.1), (65_536, 40, 1, 0, 0), (65_537, 513, 300, 0, 0), (2_100_001, 9, 100_000, 0.01, 0.02)])
@pytest.mark.parametrize("t,o,accumulate", [("f32", "f32", False), ("bf16", "f32", True), ("f16", "f16", True), ("bf16", "bf16", False)])
def test_gradients_of_many_places(n, dim, vocab, hot, padding, t, o, accumulate):
    torch, sidco = _torch(), _sidco()
    gap = n % 2 * 5
    grad, _ = _matrix(n, dim, t, 4, gap)
    w, words = _words(n, vocab, 5, n % 3 == 0, padding, hot)
    inside = torch.from_numpy(ref.inside(w, vocab)).to("cuda")
    grad[~inside] = float("nan")  # what stands in padding is not looked at
    table, whole = _matrix(vocab, dim, o, 6, gap, scale=2.0**-3)
    before, old = whole.clone(), table.double()
    sidco.sidco_embedding_grad(grad, words, table, scale=0.75, accumulate=accumulate)
    torch.cuda.synchronize()
    own, rows = words.long()[inside], grad.double()[inside]
    want, size = (torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, own, r) * 0.75 for r in (rows, rows.abs()))
    count = torch.bincount(own, minlength=vocab)
    rel, least = _half_step(o)
    # count additions, the scale (exact here) and the old value's addition, each rounded to 32 bits; the last to the result's
    bound = (count[:, None] + 2) * 2.0**-24 * size
    if accumulate:
        want = want + old
        bound = bound + 2.0**-24 * (old.abs() + size)
    bound = bound + (want.abs() + bound) * rel + least
    got = table.double()
    none = count == 0
    assert torch.equal(got[none], old[none] if accumulate else torch.zeros_like(got[none]))
    assert bool(((got - want).abs() <= bound)[~none].all()), float((got - want).abs().max())
    if gap:
        assert torch.equal(whole[:, 0], before[:, 0]) and torch.equal(whole[:, 1 + dim:], before[:, 1 + dim:])


def test_dropout_of_more_rows_than_blocks():
    torch, sidco = _torch(), _sidco()
    rows, cols = 2**20 + 77, 1025
    x = torch.ones(rows, cols, dtype=torch.float16, device="cuda")
    y = torch.empty_like(x)
    sidco.sidco_dropout(x, y, 0.25, 12, offset=5)
    for r in (0, 2**19, 2**20 - 40, 2**20 + 37):
        kept = torch.from_numpy(ref.numbers(40, cols, 12, 5 + sidco.sidco_dropout_blocks(r, cols) if r else 5) >= 16384).to("cuda")
        assert torch.equal(y[r:r + 40] != 0, kept), r
