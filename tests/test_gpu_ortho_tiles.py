"""GPU: the orthogonalised update of sizes that take each of the tiles, one launch and two for X, and groups of steps: wide and
tall, with row strides, every precision and type of result, random matrices, matrices that lack directions, and NaN.  The
reference is the definition in 64 bits.  test_dense_plans.py checks that these sizes take what they are here for.

Bounds as in test_gpu_ortho_spectra.py, where halves are not taken throughout.  With halves throughout (precision 1): random
matrices 5e-3; of rank 32, whose result has the norm 32^0.5, what the first X, of norm 1, and the first G and P lose by
rounding to 11 bits (0.6 * 2^-11 each in the mean of squares) grows by 3.4445^5: 0.6 * 2^-11 * 485 * (3 / 32)^0.5 = 4.4e-2.  Sums are of up to
9000 terms in fp32: at most 9000^0.5 * 2^-24 of a sum in the mean, far below either."""
import functools

import pytest

from test_gpu_ortho import COEF, ROUNDING

pytestmark = pytest.mark.gpu

# batch, rows, columns (and exchanged)
SHAPES = [(6, 256, 2304), (8, 701, 3001), (4, 1501, 6001), (8, 1499, 1599), (1, 2001, 9003), (2, 3701, 3805)]
KINDS = [("float32", 0), ("float16", 0), ("bfloat16", 0), ("bfloat16", 2), ("float32", 1), ("float16", 1), ("bfloat16", 1)]
RANDOM, LACKING = 0, 1
BOUND = {("float32", 0): (1.8e-4, 1.8e-4), ("float16", 0): (1.8e-4, 1.8e-4), ("bfloat16", 0): (3.1e-3, 3.1e-3), ("bfloat16", 2): (1.8e-4, 1.8e-4),
         ("float32", 1): (5e-3, 4.4e-2), ("float16", 1): (5e-3, 4.4e-2), ("bfloat16", 1): (5e-3, 4.4e-2)}


def _torch():
    import torch
    return torch


def _sidco():
    import paper_2101_10761_amd as sidco
    return sidco


def newton_schulz(x, steps=5, coef=COEF, eps=1e-7):
    """The definition, on the GPU in 64 bits."""
    torch = _torch()
    a, b, c = coef
    tall = x.shape[0] > x.shape[1]
    x = x.double()
    x = (x.t() if tall else x).contiguous()
    x = x / (x.square().sum().sqrt() + eps)
    for _ in range(steps):
        g = x @ x.t().contiguous()
        x = a * x + (b * g + c * torch.mm(g, g)) @ x
    return x.t() if tall else x


def _matrices(batch, rows, cols):
    """Random, of rank 32, then random ones of other sizes; with three or more the last one holds a NaN."""
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = normal(batch, rows, cols) * 1e-3
    if batch > 1:
        x[1] = normal(rows, 32) @ normal(32, cols)
    if batch > 2:
        x[batch - 1, rows - 1, cols - 1] = float("nan")
    return x


@functools.lru_cache(maxsize=1)
def _case(batch, rows, cols):
    x = _matrices(batch, rows, cols)
    return x, [newton_schulz(x[z]) for z in range(min(batch, 3))]


def _off(got, want):
    return float((got.double() - want).norm() / want.norm())


def _check(out, want, batch, dtype, precision):
    for z, w in enumerate(want):
        if z > 1 and z == batch - 1:
            break
        bound = BOUND[dtype, precision][LACKING if z == 1 else RANDOM] + ROUNDING[dtype]
        assert _off(out[z], w) <= bound, z
    if batch > 2:
        assert bool(out[batch - 1].isnan().all())
        assert not bool(out[:batch - 1].isnan().any())


@pytest.mark.parametrize("batch,rows,cols", [s for b, m, n in SHAPES for s in ((b, m, n), (b, n, m))])
@pytest.mark.parametrize("dtype,precision", KINDS)
def test_matrices(batch, rows, cols, dtype, precision):
    torch, sidco = _torch(), _sidco()
    x, want = _case(batch, rows, cols)
    buf = torch.full((batch, rows + 1, cols + 3), 7.0, dtype=getattr(torch, dtype), device="cuda")
    out = buf[:, 1:, 1:cols + 1]
    sidco.sidco_orthogonalize(x, out, precision=precision)
    _check(out, want, batch, dtype, precision)
    out.fill_(7.0)
    assert bool((buf == 7.0).all()), "written outside the result"


@pytest.mark.parametrize("batch,rows,cols", [s for b, m, n in SHAPES[:4] for s in ((b, m, n), (b, n, m))])
@pytest.mark.parametrize("grad_dtype,weight_dtype", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float16")])
def test_steps(batch, rows, cols, grad_dtype, weight_dtype):
    torch, sidco = _torch(), _sidco()
    g = _matrices(batch, rows, cols).to(getattr(torch, grad_dtype))
    gen = torch.Generator(device="cuda").manual_seed(3)
    m = torch.randn(g.shape, generator=gen, device="cuda") * 1e-3
    w = (torch.randn(g.shape, generator=gen, device="cuda") / cols ** 0.5).to(getattr(torch, weight_dtype))
    m0, w0 = m.clone(), w.clone()
    lr, mu, decay = 0.05, 0.9, 0.1
    sidco.sidco_muon_step(g, m, w, lr=lr, mu=mu, weight_decay=decay)
    f = lambda v: float(_torch().tensor(v, dtype=torch.float32))  # noqa: E731
    for z in range(min(batch - 1, 2)):
        moved = f(mu) * m0[z].double() + g[z].double()
        assert float((m[z].double() - moved).abs().max()) <= 2.0 ** -22 * float(moved.abs().max() + g[z].double().abs().max())
        update = newton_schulz(g[z].double() + f(mu) * m[z].double())
        want = (1 - f(lr) * f(decay)) * w0[z].double() - f(lr) * update
        room = max(BOUND[weight_dtype, 0]) * lr * float(update.norm()) + (ROUNDING[weight_dtype] + 2.0 ** -22) * float(w0[z].double().norm() + lr * update.norm())
        assert float((w[z].double() - want).norm()) <= room, z
    if batch > 2:
        assert bool(w[batch - 1].isnan().all()) and not bool(w[:batch - 1].isnan().any())


@pytest.mark.parametrize("coef,steps", [((4.0, -6.6, 2.75), 3), ((4.0, -6.6, 2.75), 5), ((4.5, -8.4, 3.5), 2), ((4.5, -8.4, 3.5), 5),
                                        ((1.5, -0.5, 0.0), 4), ((1.5, -0.5, 0.0), 9)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_other_coefficients_and_steps_in_groups(coef, steps, dtype):
    """A step multiplies by up to another a: 3 * 2^-23 * a^steps in place of the 1.8e-4, and before a result in bf16, where a
    is at most 4, the last step's halves."""
    torch, sidco = _torch(), _sidco()
    batch, rows, cols = SHAPES[0]
    x, _ = _case(batch, rows, cols)
    out = torch.empty((2, rows, cols), dtype=getattr(torch, dtype), device="cuda")
    sidco.sidco_orthogonalize(x[2:4], out, steps=steps, coef=coef)
    for z in range(2):
        bound = max(1.8e-4, 3 * 2.0 ** -23 * coef[0] ** steps) + (3.1e-3 * 4.0 / 3.4445 if dtype == "bfloat16" else 0.0)
        assert _off(out[z], newton_schulz(x[2 + z], steps, coef)) <= bound + ROUNDING[dtype]
