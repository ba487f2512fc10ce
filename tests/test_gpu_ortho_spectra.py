"""GPU: the orthogonalised update of matrices whose singular values are not alike, as momenta's are not.

Bounds (2-norm of the difference over 2-norm of the result), with COEF's a = 3.4445 the largest that a step multiplies by:
  result in bf16  its own rounding, 2^-9; and the last step's operands in 11 bits: X, G and P each off by at most 2^-11 an element,
                  0.6 of it in the mean of squares, independent of each other, times 3.4445, on singular values that the step takes
                  from at most 1.2 to at least 0.7: 2^-9 + sqrt(3) * 0.6 * 2^-11 * 3.4445 * 1.2 / 0.7 = 5e-3
  result in fp16  its own rounding, 2^-11, and 22 bits throughout: what the first roundings leave in directions that the matrix
                  lacks grows by 3.4445 a step, 3 * 2^-23 * 3.4445^5 = 1.8e-4
  result in fp32  the 1.8e-4 alone"""
import numpy as np
import pytest

import dense_reference as ref
from test_gpu_ortho import COEF, _dev, _host, _off, _sidco, _torch

pytestmark = pytest.mark.gpu

BOUND = {"bfloat16": 5e-3, "float16": 2.0 ** -11 + 1.8e-4, "float32": 1.8e-4}
SPECTRA = {
    "flat": lambda k: np.ones(len(k)),
    "1/k": lambda k: 1.0 / k,
    "1/k^2": lambda k: 1.0 / k ** 2,
    "exponential": lambda k: np.exp(-k / 10.0),
    "rank 32": lambda k: (k <= 32).astype(float),
    "rank 1": lambda k: (k <= 1).astype(float),
}


def with_spectrum(rng, rows, cols, spectrum):
    m, n = min(rows, cols), max(rows, cols)
    u = np.linalg.qr(rng.standard_normal((m, m)))[0]
    v = np.linalg.qr(rng.standard_normal((n, m)))[0].T
    x = (u * SPECTRA[spectrum](np.arange(1, m + 1))) @ v
    return (x if rows <= cols else x.T).astype(np.float32)


# one block a matrix; single steps; a group of steps, wide and tall, one tile and several
@pytest.mark.parametrize("rows,cols", [(60, 500), (65, 300), (150, 100), (128, 2000), (1400, 200), (256, 1024)])
@pytest.mark.parametrize("spectrum", list(SPECTRA))
@pytest.mark.parametrize("dtype", list(BOUND))
def test_spectra(rows, cols, spectrum, dtype):
    torch, sidco = _torch(), _sidco()
    x = with_spectrum(np.random.default_rng(rows + cols), rows, cols, spectrum)
    out = torch.empty((rows, cols), dtype=getattr(torch, dtype), device="cuda")
    sidco.sidco_orthogonalize(_dev(x), out)
    off = _off(_host(out), ref.newton_schulz(x, 5, COEF, 1e-7))
    assert off <= BOUND[dtype], off


@pytest.mark.parametrize("rows,cols", [(60, 500), (200, 1300), (1400, 200)])
def test_step_of_a_low_rank_gradient(rows, cols):
    """Weights in bf16, zero before the step, so that they are the update itself."""
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(rows)
    g = _dev(np.stack([with_spectrum(rng, rows, cols, s) for s in ("rank 32", "1/k^2")]))
    m, w = torch.zeros_like(g), torch.zeros(g.shape, dtype=torch.bfloat16, device="cuda")
    sidco.sidco_muon_step(g, m, w, lr=0.5, mu=0.9)
    for z in range(2):
        want = -0.5 * ref.newton_schulz(_host(g[z]) * 1.9, 5, COEF, 1e-7)
        assert _off(_host(w[z]), want) <= BOUND["bfloat16"]
