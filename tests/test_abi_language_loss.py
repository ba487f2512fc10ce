"""CPU: refusals of cross entropy's gradient from the losses, before any HIP call."""
import ctypes as C

from test_abi_language import OK, OTHER, _refuses, lib  # noqa: F401


def test_refusals(lib):  # noqa: F811
    good = dict(stream=None, x=OK, w=OTHER, t=0, n=5, dim=20, vocab=10, ldx=20, ldw=20, words=OK, wt=0, loss=OK, lse=OK, g=None, dx=C.c_void_p(1 << 14), ldgx=20,
                dw=C.c_void_p(1 << 15), dt=0, ldgw=20, acc=0)
    _refuses(lib.sidco_cross_entropy_grad_of_loss, good, [
        (-1, [dict(x=None), dict(w=None), dict(words=None), dict(lse=None), dict(dx=None, dw=None)]),
        (-2, [dict(n=0), dict(n=2**22 + 1), dict(dim=0), dict(vocab=0), dict(ldx=19), dict(ldw=19), dict(ldgx=19), dict(ldgw=19)]),
        (-8, [dict(loss=C.c_void_p(4098)), dict(lse=C.c_void_p(4098)), dict(g=C.c_void_p(4098)), dict(dx=C.c_void_p(4098))]),
        (-9, [dict(t=3), dict(wt=2), dict(dt=2), dict(acc=2), dict(dx=OK), dict(dw=OTHER), dict(dw=C.c_void_p(1 << 14))])])
