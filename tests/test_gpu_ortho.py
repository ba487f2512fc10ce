"""GPU: the orthogonalised update against its definition in 64 bits.

Bounds (2-norm of the difference over 2-norm of the result).  A step rounds X, G and P once each and sums in fp32; its error
is carried on by the steps after it, which move no part of X by more than they move the bulk of it by a factor of about two.
Operands of 11 bits: 2^-12 an element, three roundings and five steps, at most about 5e-3 in the worst order; of 22 bits and
fp32 sums of up to 2500 terms: 2^-20 in place of 2^-12, 2e-5.  A result of 16 bits adds its own rounding.
That factor holds for matrices whose singular values are alike.  Where u lacks directions altogether, what the roundings leave
in them grows by 3.4445 a step while the others stay near 1: 3 * 2^-12 * 3.4445^5 = 0.36 against a result of rank one, and 3 *
2^-23 * 3.4445^5 = 1.8e-4 with operands of 22 bits."""
import numpy as np
import pytest

import dense_reference as ref

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)
HALF_BOUND, FULL_BOUND = 5e-3, 2e-5
ROUNDING = {"float32": 0.0, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


def _torch():
    import torch
    return torch


def _sidco():
    import paper_2101_10761_amd as sidco
    return sidco


def _dev(a, dtype="float32"):
    torch = _torch()
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(getattr(torch, dtype))


def _host(t):
    return t.to(_torch().float64).cpu().numpy()


def _off(got, want):
    n = np.linalg.norm(want)
    return np.linalg.norm(got - want) / n if n else np.linalg.norm(got)


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (16, 20), (31, 31), (64, 576), (65, 64), (100, 1000), (300, 40), (257, 513), (500, 500), (129, 2000), (1100, 700)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("precision", [1, 2])
def test_one_matrix(rows, cols, precision):
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(rows * 31 + cols)
    x = (rng.standard_normal((rows, cols)) * 1e-3).astype(np.float32)
    want = ref.newton_schulz(x, 5, COEF, 1e-7)
    guard = torch.full((rows + 2, cols + 5), 7.0, dtype=torch.float32, device="cuda")
    out = guard[1:rows + 1, 3:cols + 3]
    sidco.sidco_orthogonalize(_dev(x), out, precision=precision)
    assert _off(_host(out), want) <= (HALF_BOUND if precision == 1 else FULL_BOUND)
    out.fill_(7.0)
    assert bool((guard == 7.0).all()), "written outside the result"


@pytest.mark.parametrize("in_dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("out_dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows,cols", [(70, 200), (200, 70)])
def test_types_and_strides(rows, cols, in_dtype, out_dtype):
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(7)
    big = _dev(rng.standard_normal((3, rows + 3, cols + 9)).astype(np.float32), in_dtype)
    x = big[:, 2:rows + 2, 5:cols + 5]
    buf = torch.full((3, rows + 1, cols + 3), 7.0, dtype=getattr(torch, out_dtype), device="cuda")
    out = buf[:, 1:, 1:cols + 1]
    sidco.sidco_orthogonalize(x, out)
    bound = (FULL_BOUND if out_dtype == "float32" else HALF_BOUND) + ROUNDING[out_dtype]
    for z in range(3):
        assert _off(_host(out[z]), ref.newton_schulz(_host(x[z]), 5, COEF, 1e-7)) <= bound
    out.fill_(7.0)
    assert bool((buf == 7.0).all())


def test_in_place_and_repeatable():
    torch, sidco = _torch(), _sidco()
    x = _dev(np.random.default_rng(1).standard_normal((5, 130, 90)).astype(np.float32))
    a, b = torch.empty_like(x), x.clone()
    sidco.sidco_orthogonalize(x, a)
    sidco.sidco_orthogonalize(b, b)
    assert torch.equal(a, b)


@pytest.mark.parametrize("precision", [1, 2])
@pytest.mark.parametrize("shape", [(60, 200), (150, 100), (400, 600)])
def test_matrices_apart(shape, precision):
    """In one batch: zeros, one nonzero element, rank one, orthonormal rows, huge, tiny, a NaN, an infinity - each as alone."""
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(2)
    n = rng.standard_normal(shape)
    one = np.zeros(shape)
    one[3, 5] = -2.0
    rank = np.outer(rng.standard_normal(shape[0]), rng.standard_normal(shape[1]))
    q = np.linalg.qr(n if shape[0] > shape[1] else n.T)[0]
    q = q if shape[0] > shape[1] else q.T
    nan, inf = n.copy(), n.copy()
    nan[shape[0] - 1, 0] = np.nan
    inf[0, shape[1] - 1] = -np.inf
    x = np.stack([np.zeros(shape), one, rank, q, n * 1e30, n * 1e-30, nan, inf, n]).astype(np.float32)
    out = torch.empty(x.shape, dtype=torch.float32, device="cuda")
    sidco.sidco_orthogonalize(_dev(x), out, eps=1e-35, precision=precision)
    got = _host(out)
    assert np.all(got[0] == 0)
    for z in (1, 2, 3, 4, 5, 8):
        want = ref.newton_schulz(x[z].astype(np.float64), 5, COEF, 1e-35)
        bound = {1: (HALF_BOUND, 0.36), 2: (FULL_BOUND, 1.8e-4)}[precision][z == 2]
        assert _off(got[z], want) <= bound, z
    assert np.all(np.isnan(got[6])) and np.all(np.isnan(got[7]))


def test_other_coefficients_and_steps():
    """The cubic iteration, many steps: the result's rows are orthonormal."""
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(3)
    x = rng.standard_normal((48, 333)).astype(np.float32)
    out = torch.empty((48, 333), dtype=torch.float32, device="cuda")
    sidco.sidco_orthogonalize(_dev(x), out, steps=20, coef=(1.5, -0.5, 0.0))
    got = _host(out)
    assert np.abs(got @ got.T - np.eye(48)).max() <= 20 * FULL_BOUND
    for steps in (1, 2, 7):
        sidco.sidco_orthogonalize(_dev(x), out, steps=steps)
        assert _off(_host(out), ref.newton_schulz(x, steps, COEF, 1e-7)) <= FULL_BOUND * max(1, steps / 5)


@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (3, 64, 100), (2, 200, 90), (6, 33, 65), (1, 700, 300)])
@pytest.mark.parametrize("grad_dtype,weight_dtype", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("bfloat16", "float16")])
@pytest.mark.parametrize("nesterov", [True, False])
def test_optimiser_step(batch, rows, cols, grad_dtype, weight_dtype, nesterov):
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(batch + rows + cols)
    shape = (batch, rows, cols)
    g = _dev((rng.standard_normal(shape) * 1e-2).astype(np.float32), grad_dtype)
    m = _dev((rng.standard_normal(shape) * 1e-1).astype(np.float32))
    w = _dev(rng.standard_normal(shape).astype(np.float32) / np.sqrt(cols), weight_dtype)
    lr, mu, decay, scale = 0.05, 0.9, 0.1, 0.7
    m0, w0, g0 = _host(m), _host(w), _host(g)
    for _ in range(2):
        sidco.sidco_muon_step(g, m, w, lr=lr, mu=mu, nesterov=nesterov, weight_decay=decay, scale=scale)
        f = lambda v: float(np.float32(v))  # noqa: E731
        m1 = f(mu) * m0 + g0
        assert np.all(np.abs(_host(m) - m1) <= 2.0 ** -23 * (np.abs(m1) + np.abs(g0)) + 1e-38)
        u = g0 + f(mu) * _host(m) if nesterov else _host(m)
        bound = FULL_BOUND if weight_dtype == "float32" else HALF_BOUND
        for z in range(batch):
            o = ref.newton_schulz(u[z], 5, COEF, 1e-7)
            want = (1 - f(lr) * f(decay)) * w0[z] - f(lr) * f(scale) * o
            room = bound * lr * scale * np.linalg.norm(o) + (ROUNDING[weight_dtype] + 2.0 ** -22) * np.linalg.norm(w0[z])
            assert np.linalg.norm(_host(w[z]) - want) <= room
        m0, w0 = _host(m), _host(w)


def test_streams_and_graph():
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(4)
    xs = [_dev(rng.standard_normal((2, 150, 260)).astype(np.float32)) for _ in range(6)]
    want = []
    for x in xs:
        y = torch.empty_like(x)
        sidco.sidco_orthogonalize(x, y)
        want.append(y)
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.empty_like(x) for x in xs]
    torch.cuda.synchronize()
    for i, x in enumerate(xs):
        with torch.cuda.stream(streams[i % 3]):
            sidco.sidco_orthogonalize(x, outs[i])
    torch.cuda.synchronize()
    for o, e in zip(outs, want):
        assert torch.equal(o, e)
    x, y = xs[0].clone(), torch.empty_like(xs[0])
    side = streams[0]
    sidco.sidco_reserve(sidco.sidco_workspace_bytes_orthogonalize(2, 150, 260, sidco.GRAD_F32), stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sidco.sidco_orthogonalize(x, y, stream=side)
    for i in (1, 2, 3, 4):
        x.copy_(xs[i])
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i])
        _ = (xs[i][0] @ xs[i][1].t()).sum().item()


def test_a_callers_workspace_and_other_calls_in_it():
    """The same workspace serves the sparsifier in between, and too small a one is refused."""
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(6)
    x = _dev(rng.standard_normal((40, 300)).astype(np.float32))
    y, z = torch.empty_like(x), torch.empty_like(x)
    sidco.sidco_orthogonalize(x, y)
    d = 50_000
    need = max(sidco.sidco_workspace_bytes(d), sidco.sidco_workspace_bytes_orthogonalize(1, 40, 300, sidco.GRAD_F32))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    g = _dev(rng.laplace(0, 1e-3, d).astype(np.float32))
    cap = sidco.sidco_out_capacity(d, 0.01)
    outs = lambda: (torch.zeros(cap, dtype=torch.int32, device="cuda"), torch.zeros(cap, device="cuda"),  # noqa: E731
                    torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda"))
    a, b = outs(), outs()
    sidco.sidco_compress(g, None, 0.01, sidco.DIST_EXP, 2, *a)
    try:
        sidco.sidco_set_workspace(ws)
        sidco.sidco_orthogonalize(x, z)
        sidco.sidco_compress(g, None, 0.01, sidco.DIST_EXP, 2, *b)
        sidco.sidco_orthogonalize(x, z)
        with pytest.raises(sidco.SidcoError):
            big = torch.zeros((3000, 3000), device="cuda")
            sidco.sidco_orthogonalize(big, big)
    finally:
        torch.cuda.synchronize()
        sidco.sidco_set_workspace(None)
    assert torch.equal(y, z)
    assert int(a[2]) == int(b[2])
    assert set(a[0][:int(a[2])].tolist()) == set(b[0][:int(b[2])].tolist())


def test_binding_refuses():
    torch, sidco = _torch(), _sidco()
    x = torch.zeros((10, 30), device="cuda")
    with pytest.raises(TypeError):
        sidco.sidco_orthogonalize(x.double(), x)
    with pytest.raises(TypeError):
        sidco.sidco_orthogonalize(x.t(), x.t())
    with pytest.raises(ValueError):
        sidco.sidco_orthogonalize(x, torch.zeros((30, 10), device="cuda"))
    with pytest.raises(sidco.SidcoError):
        sidco.sidco_orthogonalize(x, x, steps=0)
    with pytest.raises(sidco.SidcoError):
        sidco.sidco_orthogonalize(x, x, eps=float("nan"))
    with pytest.raises(ValueError):
        sidco.sidco_muon_step(x, torch.zeros((10, 31), device="cuda"), x.clone(), lr=0.1)
    with pytest.raises(sidco.SidcoError):
        sidco.sidco_muon_step(x, x, x.clone(), lr=0.1)
