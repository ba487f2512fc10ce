"""Host-side checks of the dense operators that need no GPU: sizes, defaults, struct layout, and arguments refused before any
HIP call."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

import dense_reference as ref
import paper_2101_10761_amd as sidco
from paper_2101_10761_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK = C.c_void_p(4096)  # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2101_10761_amd import build
        build.build()
    return sidco.load()


def test_sizes(lib):
    for rows, cols, lines in ((1, 1, 1), (1, 256, 1), (3, 257, 6), (1, 138_357_544, 540_460), (700, 1500, 4200)):
        assert sidco.sidco_mx4_code_bytes(rows, cols) == 128 * lines
        assert sidco.sidco_mx4_scale_bytes(rows, cols) == 8 * lines
    for rows, cols in ((0, 1), (1, 0), (-1, 5), (1, 2 ** 31)):
        with pytest.raises(sidco.SidcoError):
            sidco.sidco_mx4_code_bytes(rows, cols)
        with pytest.raises(sidco.SidcoError):
            sidco.sidco_mx4_scale_bytes(rows, cols)
    base = sidco.sidco_workspace_bytes_mx4_linear(1, 1) - 136
    assert sidco.sidco_workspace_bytes_mx4_linear(20, 1500) == base + 20 * 6 * 136
    assert sidco.sidco_workspace_bytes_mx4_linear(0, 5) == 0 and sidco.sidco_workspace_bytes_mx4_linear(5, 2 ** 24 + 1) == 0
    half = sidco.sidco_workspace_bytes_orthogonalize(2, 300, 500, sidco.GRAD_BF16)
    full = sidco.sidco_workspace_bytes_orthogonalize(2, 300, 500, sidco.GRAD_F32)
    assert 0 < half < full == sidco.sidco_workspace_bytes_orthogonalize(2, 300, 500, sidco.GRAD_BF16, sidco.NS_FULL)
    assert sidco.sidco_workspace_bytes_orthogonalize(2, 500, 300, sidco.GRAD_F32) == full
    assert sidco.sidco_workspace_bytes_orthogonalize(0, 3, 3, 0) == 0
    assert sidco.sidco_workspace_bytes_orthogonalize(1, 3, 3, 7) == 0
    assert sidco.sidco_workspace_bytes_orthogonalize(1, 3, 2 ** 21 + 1, 0) == 0


def test_newton_schulz_struct(lib, tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sidco.h"\n'
                   'int main(void){printf("%zu %zu %zu %zu\\n", sizeof(sidco_newton_schulz), offsetof(sidco_newton_schulz,a),'
                   'offsetof(sidco_newton_schulz,eps), offsetof(sidco_newton_schulz,precision));return 0;}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    S = binding.NewtonSchulz
    assert got == [C.sizeof(S), S.a.offset, S.eps.offset, S.precision.offset]
    d = sidco.sidco_newton_schulz_default()
    assert (d.steps, d.precision) == (5, 0)
    assert (d.a, d.b, d.c) == tuple(float(np.float32(v)) for v in (3.4445, -4.7750, 2.0315)) and d.eps == np.float32(1e-7)


def _refuses(fn, good, wrong):
    names = list(good)
    for code, changes in wrong:
        for change in changes:
            args = dict(good, **change)
            assert fn(*[args[n] for n in names]) == code, (change, code)


def test_exchange_refusals(lib):
    good = dict(stream=None, grad=OK, t=0, residual=C.c_void_p(8192), d=1000, codes=OK, scales=OK)
    _refuses(lib.sidco_mx4_compress, good, [
        (-1, [dict(grad=None), dict(codes=None), dict(scales=None)]),
        (-2, [dict(d=0), dict(d=-3), dict(d=2 ** 31)]),
        (-8, [dict(grad=C.c_void_p(4098)), dict(t=2, grad=C.c_void_p(4097)), dict(residual=C.c_void_p(8193)),
              dict(codes=C.c_void_p(4104)), dict(scales=C.c_void_p(4100))]),
        (-9, [dict(t=3), dict(t=-1), dict(residual=OK)])])
    good = dict(stream=None, codes=OK, cs=512, scales=OK, ss=32, workers=3, d=1000, scale=1.0, acc=0, dense=C.c_void_p(8192))
    _refuses(lib.sidco_mx4_aggregate, good, [
        (-1, [dict(codes=None), dict(scales=None), dict(dense=None)]),
        (-2, [dict(d=0), dict(d=2 ** 31), dict(workers=0), dict(cs=496), dict(ss=24), dict(cs=-512)]),
        (-8, [dict(codes=C.c_void_p(4104)), dict(scales=C.c_void_p(4097)), dict(dense=C.c_void_p(8194)), dict(cs=520), dict(ss=36)]),
        (-9, [dict(scale=math.nan), dict(scale=math.inf), dict(acc=2), dict(acc=-1)])])


def test_matrix_refusals(lib):
    good = dict(stream=None, x=OK, t=0, rows=10, cols=20, ld=20, codes=OK, scales=OK, codes_t=OK, scales_t=OK)
    _refuses(lib.sidco_mx4_quantize, good, [
        (-1, [dict(x=None), dict(codes=None), dict(scales=None), dict(codes_t=None), dict(scales_t=None),
              dict(codes=None, scales=None, codes_t=None, scales_t=None)]),
        (-2, [dict(rows=0), dict(cols=0), dict(ld=19), dict(rows=2 ** 31), dict(ld=2 ** 31),
              dict(rows=2 ** 31 - 1, cols=2 ** 31 - 1, ld=2 ** 31 - 1)]),
        (-8, [dict(x=C.c_void_p(4098)), dict(codes=C.c_void_p(4104)), dict(scales=C.c_void_p(4100)),
              dict(codes_t=C.c_void_p(4104)), dict(scales_t=C.c_void_p(4100))]),
        (-9, [dict(t=3)])])
    good = dict(stream=None, codes=OK, scales=OK, rows=10, cols=20, out=OK, t=0, ld=20)
    _refuses(lib.sidco_mx4_dequantize, good, [
        (-1, [dict(out=None), dict(codes=None), dict(scales=None)]),
        (-2, [dict(rows=0), dict(cols=0), dict(ld=19), dict(rows=2 ** 31), dict(ld=2 ** 31)]),
        (-8, [dict(out=C.c_void_p(4098)), dict(codes=C.c_void_p(4104)), dict(scales=C.c_void_p(4100))]),
        (-9, [dict(t=3)])])


def test_product_refusals(lib):
    good = dict(stream=None, a=OK, sa=OK, b=OK, sb=OK, m=10, n=20, k=30, alpha=1.0, acc=0, c=OK, t=0, ld=20)
    result = [
        (-1, [dict(c=None)]),
        (-2, [dict(n=0), dict(n=2 ** 31), dict(k=0), dict(k=2 ** 24 + 1), dict(ld=19), dict(ld=2 ** 31)]),
        (-8, [dict(c=C.c_void_p(4098)), dict(t=1, c=C.c_void_p(4097))]),
        (-9, [dict(t=3), dict(alpha=math.nan), dict(acc=2)])]
    _refuses(lib.sidco_mx4_matmul, good, result + [
        (-1, [dict(a=None), dict(sa=None), dict(b=None), dict(sb=None)]),
        (-2, [dict(m=0), dict(m=2 ** 31), dict(m=2 ** 31 - 1, n=2 ** 31 - 1, ld=2 ** 31 - 1)]),
        (-8, [dict(a=C.c_void_p(4104)), dict(sa=C.c_void_p(4100)), dict(b=C.c_void_p(4104)), dict(sb=C.c_void_p(4100))])])
    good = dict(stream=None, x=OK, xt=0, rows=10, k=30, ldx=30, b=OK, sb=OK, n=20, alpha=1.0, acc=0, c=OK, t=0, ld=20)
    _refuses(lib.sidco_mx4_linear, good, result + [
        (-1, [dict(x=None), dict(b=None), dict(sb=None)]),
        (-2, [dict(rows=0), dict(rows=2 ** 31), dict(ldx=29), dict(ldx=2 ** 31)]),
        (-8, [dict(x=C.c_void_p(4098)), dict(b=C.c_void_p(4104)), dict(sb=C.c_void_p(4100))]),
        (-9, [dict(xt=3)])])


def test_orthogonalize_refusals(lib):
    def opt(**kw):
        o = sidco.sidco_newton_schulz_default()
        for k, v in kw.items():
            setattr(o, k, v)
        return C.byref(o)
    bad_opt = [(-4, [dict(opt=opt(steps=0)), dict(opt=opt(steps=101))]),
               (-9, [dict(opt=opt(a=math.nan)), dict(opt=opt(b=math.inf)), dict(opt=opt(c=math.nan)), dict(opt=opt(eps=-1.0)),
                     dict(opt=opt(eps=math.nan)), dict(opt=opt(precision=3))])]
    good = dict(stream=None, x=OK, xt=0, ldx=20, xs=200, batch=2, rows=10, cols=20, opt=None, out=OK, t=0, ldo=20, os=200)
    _refuses(lib.sidco_orthogonalize, good, bad_opt + [
        (-1, [dict(x=None), dict(out=None)]),
        (-2, [dict(batch=0), dict(batch=65536), dict(rows=0), dict(cols=0), dict(rows=2 ** 21 + 1), dict(ldx=19), dict(ldo=19),
              dict(xs=199), dict(os=199), dict(batch=65535, rows=2 ** 21, cols=2 ** 21, ldx=2 ** 21, ldo=2 ** 21)]),
        (-8, [dict(x=C.c_void_p(4098)), dict(out=C.c_void_p(4097), t=2)]),
        (-9, [dict(xt=3), dict(t=-1)])])
    good = dict(stream=None, g=OK, gt=0, m=C.c_void_p(8192), w=C.c_void_p(16384), wt=0, batch=2, rows=10, cols=20, lr=0.1, mu=0.9,
                nesterov=1, decay=0.0, scale=1.0, opt=None)
    _refuses(lib.sidco_muon_step, good, bad_opt + [
        (-1, [dict(g=None), dict(m=None), dict(w=None)]),
        (-2, [dict(batch=0), dict(rows=0), dict(cols=2 ** 21 + 1)]),
        (-8, [dict(g=C.c_void_p(4098)), dict(m=C.c_void_p(8194)), dict(w=C.c_void_p(16386))]),
        (-9, [dict(gt=3), dict(wt=3), dict(lr=math.nan), dict(mu=math.inf), dict(decay=math.nan), dict(scale=math.nan), dict(nesterov=2),
              dict(m=OK), dict(w=OK), dict(w=C.c_void_p(8192))])])


def test_reference_by_hand():
    """The reference itself: blocks worked out by hand, and the limits of the iteration."""
    x = np.zeros((1, 64))
    x[0, :8] = [4, 6, 7.9, -0.25, 0.75, 2.5, 3.5, 5]   # largest 7.9: e = 2, unit 1
    x[0, 32:36] = [1.0, 0.9, 0.1, -0.07]               # largest 1: e = 0, unit 1/4
    code, byte = ref.mx4_blocks(x)
    assert byte[0, 0] == 127 and byte[0, 1] == 125
    assert code[0, :8].tolist() == [6, 7, 7, 8, 2, 4, 6, 6]
    assert ref.mx4_values(code, byte, 64)[0, 32:36].tolist() == [1.0, 1.0, 0.125, -0.125]
    assert ref.mx4_blocks(np.full((1, 1), 1e-45))[1][0, 0] == 0
    assert ref.mx4_blocks(np.full((1, 1), np.nan))[1][0, 0] == 255
    q = np.linalg.qr(np.random.default_rng(0).standard_normal((9, 4)))[0]
    s = 0.5  # |q| = 2: every singular value starts at one half
    for _ in range(3):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    np.testing.assert_allclose(ref.newton_schulz(q, 3, (3.4445, -4.7750, 2.0315), 0.0), s * q, atol=1e-12)
    np.testing.assert_allclose(ref.newton_schulz(q.T, 3, (3.4445, -4.7750, 2.0315), 0.0), s * q.T, atol=1e-12)
