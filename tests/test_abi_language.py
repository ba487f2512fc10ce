"""Host-side checks of a language model's operators that need no GPU: the reference by hand, sizes, and arguments refused before
any HIP call."""
import ctypes as C
import math
import os

import numpy as np
import pytest

import language_reference as ref
import paper_2101_10761_amd as sidco
from paper_2101_10761_amd import binding

OK = C.c_void_p(4096)  # never dereferenced
OTHER = C.c_void_p(8192)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2101_10761_amd import build
        build.build()
    return sidco.load()


def _refuses(fn, good, wrong):
    names = list(good)
    for code, changes in wrong:
        for change in changes:
            args = dict(good, **change)
            assert fn(*[args[n] for n in names]) == code, (change, code)


def test_the_generator_by_its_published_answers():
    """The known answers that the generator was published with."""
    assert ref.philox([0, 0, 0, 0], [0, 0]) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert ref.philox([ones] * 4, [ones] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert ref.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420,
                                                                                                    0x24126EA1]
    seed, offset = 0x123456789ABCDEF0, 2**32 - 2
    got = ref.numbers(3, 11, seed, offset)
    for r in range(3):
        for c in range(11):
            b = offset + 2 * r + c // 8
            word = ref.philox([b & ones, b >> 32, 0, 0], [seed & ones, seed >> 32])[c % 8 // 2]
            assert got[r, c] == (word >> 16 if c % 2 else word & 0xFFFF)


def test_reference_by_hand():
    table = np.arange(6.0).reshape(3, 2)
    assert ref.embedding(table, np.array([2, -1, 0, 3]), 2.0).tolist() == [[8, 10], [0, 0], [0, 2], [0, 0]]
    total, size, count = ref.embedding_grad(np.array([[1.0], [-2], [5], [7]]), np.array([1, 1, -1, 2]), 3, 0.5)
    assert total.tolist() == [[0], [-0.5], [3.5]] and size.tolist() == [[0], [1.5], [3.5]] and count.tolist() == [0, 2, 1]


def test_sizes(lib):
    assert sidco.sidco_dropout_blocks(3, 8) == 3 and sidco.sidco_dropout_blocks(3, 9) == 6
    assert sidco.sidco_dropout_blocks(2**31 - 1, 2**31 - 1) == (2**31 - 1) * 2**28
    for rows, cols in ((0, 1), (1, 0), (2**31, 1)):
        with pytest.raises(sidco.SidcoError):
            sidco.sidco_dropout_blocks(rows, cols)
    assert 0 < sidco.sidco_workspace_bytes_embedding_grad(1, 1) < sidco.sidco_workspace_bytes_embedding_grad(10**6, 1500)
    assert sidco.sidco_workspace_bytes_embedding_grad(0, 1) == 0 and sidco.sidco_workspace_bytes_embedding_grad(1, 2**31) == 0
    assert sidco.sidco_workspace_bytes_embedding_grad(2**27, 512) > 0 and sidco.sidco_workspace_bytes_embedding_grad(2**27 + 1, 1) == 0


def test_embedding_refusals(lib):
    words = [(-1, [dict(words=None)]),
             (-2, [dict(n=0), dict(n=2**31), dict(vocab=0), dict(vocab=2**31), dict(dim=0), dict(ldt=19), dict(ldo=19), dict(ldt=2**31)]),
             (-8, [dict(words=C.c_void_p(4098)), dict(wt=1, words=C.c_void_p(4100))]),
             (-9, [dict(wt=2), dict(wt=-1), dict(t=3), dict(ot=-1), dict(scale=math.nan), dict(scale=math.inf)])]
    good = dict(stream=None, table=OK, t=0, vocab=10, dim=20, ldt=20, words=OK, wt=0, n=5, scale=1.0, out=OTHER, ot=0, ldo=20)
    _refuses(lib.sidco_embedding, good, words + [
        (-1, [dict(table=None), dict(out=None)]),
        (-8, [dict(table=C.c_void_p(4098)), dict(ot=1, out=C.c_void_p(4097))]),
        (-9, [dict(out=OK)])])
    good = dict(stream=None, grad=OK, t=0, n=5, dim=20, ldo=20, words=OK, wt=0, vocab=10, scale=1.0, acc=0, table=OTHER, ot=0, ldt=20)
    _refuses(lib.sidco_embedding_grad, good, words + [
        (-1, [dict(table=None), dict(grad=None)]),
        (-2, [dict(n=2**31 - 1, dim=2**20, ldo=2**20, ldt=2**20), dict(n=2**27 + 1), dict(n=9, dim=2**31 - 1, ldo=2**31 - 1, ldt=2**31 - 1)]),
        (-8, [dict(grad=C.c_void_p(4098)), dict(ot=1, table=C.c_void_p(4097))]),
        (-9, [dict(acc=2), dict(acc=-1), dict(table=OK)])])


def test_dropout_refusals(lib):
    good = dict(stream=None, x=OK, t=0, rows=10, cols=20, ldx=20, p=0.5, seed=1, offset=0, more=None, res=None, ldr=20, y=OTHER, ot=0, ldy=20)
    _refuses(lib.sidco_dropout, good, [
        (-1, [dict(x=None), dict(y=None)]),
        (-2, [dict(rows=0), dict(rows=2**31), dict(cols=0), dict(ldx=19), dict(ldy=19), dict(res=OK, ldr=19), dict(ldy=2**31)]),
        (-8, [dict(x=C.c_void_p(4098)), dict(y=C.c_void_p(4097), ot=2), dict(more=C.c_void_p(4100)), dict(res=C.c_void_p(4098))]),
        (-9, [dict(t=3), dict(ot=3), dict(p=-0.1), dict(p=1.1), dict(p=math.nan), dict(y=OK, ot=1), dict(y=OK, ldy=24),
              dict(res=OTHER, ldr=24)])])


def test_cross_entropy_refusals(lib):
    good = dict(stream=None, x=OK, w=OTHER, t=0, n=5, dim=20, vocab=10, ldx=20, ldw=20, words=OK, wt=0, loss=OK, lse=OTHER)
    both = [(-1, [dict(x=None), dict(w=None), dict(words=None)]),
            (-2, [dict(n=0), dict(n=2**22 + 1), dict(dim=0), dict(dim=2**21 + 1, ldx=2**22, ldw=2**22), dict(vocab=0), dict(vocab=2**31), dict(ldx=19),
                  dict(ldw=19), dict(n=2**22, vocab=2**31 - 1), dict(vocab=2**31 - 1, dim=2**13, ldx=2**13, ldw=2**13)]),
            (-8, [dict(x=C.c_void_p(4098)), dict(t=1, w=C.c_void_p(4097)), dict(words=C.c_void_p(4098)), dict(wt=1, words=C.c_void_p(4100)),
                  dict(lse=C.c_void_p(4098))]),
            (-9, [dict(t=3), dict(t=-1), dict(wt=2)])]
    _refuses(lib.sidco_cross_entropy, good, both + [(-1, [dict(loss=None, lse=None)]), (-8, [dict(loss=C.c_void_p(4098))]), (-9, [dict(lse=OK)])])
    good = dict(stream=None, x=OK, w=OTHER, t=0, n=5, dim=20, vocab=10, ldx=20, ldw=20, words=OK, wt=0, lse=OK, g=None, dx=C.c_void_p(1 << 14), ldgx=20,
                dw=C.c_void_p(1 << 15), dt=0, ldgw=20, acc=0)
    _refuses(lib.sidco_cross_entropy_grad, good, both + [
        (-1, [dict(lse=None), dict(dx=None, dw=None)]),
        (-2, [dict(ldgx=19), dict(ldgw=19), dict(ldgw=2**31)]),
        (-8, [dict(g=C.c_void_p(4098)), dict(dx=C.c_void_p(4098)), dict(dw=C.c_void_p(4098))]),
        (-9, [dict(dt=2), dict(dt=1), dict(t=1, dt=2), dict(acc=2), dict(dx=OK), dict(dx=OTHER), dict(dw=OK), dict(dw=OTHER), dict(dw=C.c_void_p(1 << 14))])])
    assert sidco.sidco_workspace_bytes_cross_entropy(0, 5, 5, 0) == 0 and sidco.sidco_workspace_bytes_cross_entropy(5, 5, 5, 3) == 0
    assert sidco.sidco_workspace_bytes_cross_entropy_grad(5, 5, 5, 1, 2) == 0
    bytes_of = lambda t, o: sidco.sidco_workspace_bytes_cross_entropy_grad(700, 1500, 10_000, t, o)  # noqa: E731
    assert 0 < bytes_of(2, 2) < bytes_of(2, 0) < bytes_of(1, 0) == bytes_of(1, 1) < bytes_of(0, 0)


def test_reference_loss_by_hand():
    torch = pytest.importorskip("torch")
    x, w = torch.tensor([[0.0, 1.0], [2.0, 0.0], [1.0, 1.0]]), torch.tensor([[math.log(2.0), 0.0], [0.0, math.log(3.0)]])
    r = ref.CrossEntropy(x, w, torch.tensor([1, 0, -1]), torch.tensor([1.0, 0.5, 1.0]))
    # logits (0, log 3), (log 4, 0): probabilities 1/4, 3/4 and 4/5, 1/5
    assert torch.allclose(r.loss, torch.tensor([math.log(4 / 3), math.log(5 / 4), 0.0], dtype=torch.float64), atol=1e-6)
    p = torch.tensor([[0.25, -0.25], [-0.1, 0.1], [0.0, 0.0]], dtype=torch.float64)
    assert torch.allclose(r.p, p, atol=1e-6)
    assert torch.allclose(r.x_grad()[0], p @ w.double(), atol=1e-6) and torch.allclose(r.w_grad(torch.float32)[0], p.t() @ x.double(), atol=1e-6)
    assert float(r.x_grad()[1].max()) < 1e-5


def test_binding_refuses_what_is_no_tensor_of_the_card(lib):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    words = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: sidco.sidco_embedding(x, words, x), lambda: sidco.sidco_embedding(None, words, x),
                 lambda: sidco.sidco_embedding_grad(x, words, x), lambda: sidco.sidco_dropout(x, x, 0.5, 1),
                 lambda: sidco.sidco_dropout([1.0], x, 0.5, 1), lambda: sidco.sidco_cross_entropy(x, x, words, x, x),
                 lambda: sidco.sidco_cross_entropy_grad(x, x, words, x, None, x)):
        with pytest.raises(TypeError):
            call()
