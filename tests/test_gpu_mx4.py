"""GPU: 4-bit microscaled gradients, matrices and products against their definition in 64 bits.

Quantisation, its residual and what is read back are exact and compared bit for bit.  Products are compared bit for bit where
every partial sum is a whole number of units below 2^24, which fp32 holds exactly in any order, and elsewhere against a bound
on fp32 sums: k additions of relative 2^-23 each, of the sum of magnitudes."""
import numpy as np
import pytest

import dense_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["float32", "float16", "bfloat16"]


def _torch():
    import torch
    return torch


def _sidco():
    import paper_2101_10761_amd as sidco
    return sidco


def _dev(a, dtype=None):
    torch = _torch()
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda")
    return t if dtype is None else t.to(getattr(torch, dtype))


def _host(t):
    return t.to(_torch().float64).cpu().numpy()


def _packed(rows, cols):
    torch, sidco = _torch(), _sidco()
    assert sidco.sidco_mx4_code_bytes(rows, cols) == rows * (-(-cols // 256)) * 128
    assert sidco.sidco_mx4_scale_bytes(rows, cols) == rows * (-(-cols // 256)) * 8
    p = -(-cols // 256)
    return (torch.full((rows, p * 128), 0xA5, dtype=torch.uint8, device="cuda"),
            torch.full((rows, p * 8), 0xA5, dtype=torch.uint8, device="cuda"))


def _upload(x):
    """A float64 matrix of representable numbers as packed device buffers."""
    code, byte = ref.mx4_blocks(x)
    return _dev(ref.mx4_pack(code)), _dev(byte)


def _special(rng, rows, cols):
    """Values over the whole exponent range, ties, zeros, denormals, infinities and NaN."""
    x = (rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-40, 40, (rows, cols)))).astype(np.float32)
    flat = x.reshape(-1)
    n = flat.size
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 4.0, -0.25, -0.75, -2.5, -5.0, -7.9, 0.0], np.float32)
    for at in range(0, n - 32, 97):
        kind = (at // 97) % 8
        if kind == 0:
            flat[at:at + 32] = np.tile(ties, 2) * np.float32(2.0) ** rng.integers(-100, 100)
        elif kind == 1:
            flat[at:at + 32] = 0
        elif kind == 2:
            flat[at:at + 32] = rng.standard_normal(32) * 1e-40
        elif kind == 3:
            flat[at:at + 32] = rng.standard_normal(32).astype(np.float32) * np.float32(5e37)
        elif kind == 4:
            flat[at] = np.inf
        elif kind == 5:
            flat[at + 5] = -np.inf
        elif kind == 6:
            flat[at + 9] = np.nan
        else:
            flat[at] = np.float32(2.0) ** -126
    return x


def _equal(got, want, what):
    got, want = np.asarray(got), np.asarray(want)
    assert got.shape == want.shape, what
    bad = np.argwhere(got != want)
    assert bad.size == 0, f"{what}: {len(bad)} differ, first at {bad[0]}: {got[tuple(bad[0])]} and {want[tuple(bad[0])]}"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 33), (32, 32), (5, 256), (129, 257), (300, 130), (127, 1000), (700, 1500)])
def test_matrix_both_ways(rows, cols, dtype):
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(rows * 1000 + cols)
    x = _dev(_special(rng, rows, cols), dtype)
    want = _host(x)
    for along, across in ((True, True), (True, False), (False, True)):
        a, b = _packed(rows, cols), _packed(cols, rows)
        sidco.sidco_mx4_quantize(x, *(a if along else (None, None)), *(b if across else (None, None)))
        for used, (codes, scales), w in ((along, a, want), (across, b, want.T)):
            if not used:
                assert bool((codes == 0xA5).all()) and bool((scales == 0xA5).all())
                continue
            code, byte = ref.mx4_blocks(w)
            _equal(scales.cpu().numpy(), byte, "exponents")
            _equal(codes.cpu().numpy(), ref.mx4_pack(code), "codes")
    for out_dtype in TYPES:
        guard = torch.full((rows + 2, cols + 5), 7.0, dtype=getattr(torch, out_dtype), device="cuda")
        sidco.sidco_mx4_quantize(x, *a)
        sidco.sidco_mx4_dequantize(a[0], a[1], guard[1:rows + 1, 2:cols + 2])
        with np.errstate(all="ignore"):
            w = torch.from_numpy(ref.rounded(want)).to(getattr(torch, out_dtype)).to(torch.float64).numpy()
        np.testing.assert_array_equal(_host(guard[1:rows + 1, 2:cols + 2]), w)
        guard[1:rows + 1, 2:cols + 2] = 7.0
        assert bool((guard == 7.0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_matrix_inside_a_larger_one(dtype):
    """Row strides and starts that leave nothing aligned beyond the element."""
    sidco = _sidco()
    rng = np.random.default_rng(5)
    big = _dev(rng.standard_normal((260, 403)).astype(np.float32), dtype)
    for r0, c0, rows, cols in ((0, 1, 130, 129), (3, 3, 257, 400), (7, 2, 64, 64), (259, 0, 1, 403), (0, 402, 260, 1)):
        x = big[r0:r0 + rows, c0:c0 + cols]
        a, b = _packed(rows, cols), _packed(cols, rows)
        sidco.sidco_mx4_quantize(x, *a, *b)
        for (codes, scales), w in ((a, _host(x)), (b, _host(x).T)):
            code, byte = ref.mx4_blocks(w)
            _equal(scales.cpu().numpy(), byte, "exponents")
            _equal(codes.cpu().numpy(), ref.mx4_pack(code), "codes")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [1, 2, 31, 32, 33, 255, 256, 257, 5000, 100_003, 3_000_001])
def test_error_feedback(d, dtype):
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(d)
    for offset, with_residual in ((0, True), (1, True), (3, False)):
        gbuf = _dev(np.concatenate([np.zeros(offset, np.float32), _special(rng, 1, d)[0] if d < 200_000 else
                                    rng.laplace(0, 1e-3, d).astype(np.float32)]), dtype)
        g = gbuf[offset:]
        rbuf = torch.full((d + offset + 9,), 3.0, dtype=torch.float32, device="cuda")
        r = rbuf[offset:offset + d]
        r.copy_(torch.from_numpy(rng.laplace(0, 1e-4, d).astype(np.float32)))
        rest = r.cpu().numpy()
        with np.errstate(over="ignore", invalid="ignore"):
            acc = _host(g).astype(np.float32) + rest if with_residual else _host(g).astype(np.float32)
        assert acc.dtype == np.float32
        codes, scales = _packed(1, d)
        sidco.sidco_mx4_compress(g, r if with_residual else None, codes[0], scales[0])
        code, byte = ref.mx4_blocks(acc[None].astype(np.float64))
        _equal(scales.cpu().numpy(), byte, "exponents")
        _equal(codes.cpu().numpy(), ref.mx4_pack(code), "codes")
        got = r.cpu().numpy()
        if with_residual:
            v = ref.mx4_values(code, byte, d)[0]
            with np.errstate(invalid="ignore"):
                want = np.where(np.isnan(v), acc, (acc.astype(np.float64) - v).astype(np.float32))
            np.testing.assert_array_equal(got, want)
        else:
            np.testing.assert_array_equal(got, rest)
        assert bool((rbuf[:offset] == 3.0).all()) and bool((rbuf[offset + d:] == 3.0).all())


def test_nothing_is_lost_over_iterations():
    """What was sent plus what the residual holds is what came in, up to the roundings of the sums."""
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(8)
    d, steps = 40_001, 6
    r = torch.zeros(d, dtype=torch.float32, device="cuda")
    sent = torch.zeros(d, dtype=torch.float32, device="cuda")
    codes, scales = _packed(1, d)
    came = np.zeros(d)
    for _ in range(steps):
        g = rng.laplace(0, 1e-3, d).astype(np.float32)
        came += g
        sidco.sidco_mx4_compress(_dev(g), r, codes[0], scales[0])
        sidco.sidco_mx4_aggregate(codes, scales, sent, accumulate=True)
    size = np.abs(came) + steps * 0.03
    assert np.all(np.abs(_host(sent) + _host(r) - came) <= 2 * steps * 2.0 ** -24 * size)


@pytest.mark.parametrize("d", [1, 8, 250, 4097, 70_001])
@pytest.mark.parametrize("workers", [1, 2, 3, 8, 13])
def test_aggregate(d, workers):
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(d + workers)
    x = rng.laplace(0, 1e-3, (workers, d)).astype(np.float32)
    if d > 1000:
        x[workers - 1, 700] = np.nan  # one worker's block stands for NaN: so does the sum
    codes, scales = _upload(x.astype(np.float64))
    values = ref.rounded(x.astype(np.float64))
    for scale, accumulate, offset in ((1.0, False, 0), (1.0 / workers, True, 1), (-0.1, True, 3)):
        buf = torch.full((d + offset + 5,), 3.0, dtype=torch.float32, device="cuda")
        dense = buf[offset:offset + d]
        dense.copy_(torch.from_numpy(rng.standard_normal(d).astype(np.float32)))
        old = _host(dense)
        sidco.sidco_mx4_aggregate(codes, scales, dense, scale=scale, accumulate=accumulate)
        s = float(np.float32(scale))
        want = s * values.sum(0) + (old if accumulate else 0)
        bound = (workers + 2) * 2.0 ** -24 * (abs(s) * np.abs(values).sum(0) + (np.abs(old) if accumulate else 0))
        got = _host(dense)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        fine = ~np.isnan(want)
        assert np.all(np.abs(got - want)[fine] <= bound[fine])
        assert bool((buf[:offset] == 3.0).all()) and bool((buf[offset + d:] == 3.0).all())


def _whole(rng, rows, cols, spread=2):
    """Numbers that 4-bit blocks hold exactly: codes times one of a few powers of two."""
    code = ref.SIZES[rng.integers(0, 8, (rows, cols))] * rng.choice([-1.0, 1.0], (rows, cols))
    block = np.exp2(rng.integers(-spread, spread + 1, (rows, -(-cols // 32)))).repeat(32, 1)[:, :cols]
    x = code * block
    # a block's exponent follows from its largest magnitude: make that 4 or 6 of its unit
    x[:, ::32] = 6.0 * block[:, ::32]
    return x


SHAPES = [(1, 1, 1), (1, 17, 33), (2, 100, 256), (16, 16, 128), (17, 33, 257), (64, 64, 64), (65, 65, 300), (33, 500, 1500),
          (130, 200, 1000), (257, 255, 513), (700, 600, 1500), (1000, 333, 77), (2100, 2050, 320)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products_that_are_exact(m, n, k):
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(m + n + k)
    a, b = _whole(rng, m, k), _whole(rng, n, k)
    # units of 2^-2 * 0.5 * 2^-2 * 0.5 = 2^-6, at most 24 * 24 * 64 units a product: exact up to 455 columns of that size, and
    # the random ones are far smaller on average
    want = a @ b.T
    assert (np.abs(a) @ np.abs(b).T).max() * 64 < 2 ** 24
    pa, pb = _upload(a), _upload(b)
    np.testing.assert_array_equal(ref.rounded(a), a)
    for dtype, alpha, accumulate in (("float32", 1.0, False), ("float32", -0.5, True), ("bfloat16", 1.0, False), ("float16", 2.0, True)):
        buf = torch.full((m + 2, n + 3), 7.0, dtype=getattr(torch, dtype), device="cuda")
        out = buf[1:m + 1, 1:n + 1]
        old = _dev(rng.integers(-8, 9, (m, n)).astype(np.float32), dtype)
        out.copy_(old)
        sidco.sidco_mx4_matmul(*pa, *pb, k, out, alpha=alpha, accumulate=accumulate)
        w = torch.from_numpy(alpha * want + (_host(old) if accumulate else 0)).float().to(getattr(torch, dtype))
        np.testing.assert_array_equal(_host(out), _host(w))
        out.fill_(7.0)
        assert bool((buf == 7.0).all()), "written outside the result"


@pytest.mark.parametrize("rows,n,k", [(1, 1, 1), (1, 4096, 4096), (3, 1000, 700), (16, 50, 5000), (20, 777, 1500), (40, 64, 129), (64, 100, 2000),
                                      (65, 130, 513), (200, 300, 400), (513, 260, 96)])
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_on_rows_as_they_come(rows, n, k, dtype):
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(rows + n + k)
    big = _dev(rng.standard_normal((rows, k + 3)).astype(np.float32), dtype)
    x = big[:, 1:k + 1]
    w = rng.standard_normal((n, k)).astype(np.float32) / np.sqrt(k)
    pw = _upload(w.astype(np.float64))
    xq, wq = ref.rounded(_host(x)), ref.rounded(w)
    out = torch.full((rows, n), 7.0, dtype=torch.float32, device="cuda")
    sidco.sidco_mx4_linear(x, *pw, out)
    bound = k * 2.0 ** -23 * (np.abs(xq) @ np.abs(wq).T)
    assert np.all(np.abs(_host(out) - xq @ wq.T) <= bound)
    narrow = torch.empty((rows, n), dtype=getattr(torch, dtype), device="cuda")
    sidco.sidco_mx4_linear(x, *pw, narrow, alpha=0.5)
    np.testing.assert_array_equal(_host(narrow), _host((out * 0.5).to(narrow.dtype)))


# few rows against many or few, long or short rows: both kernels that serve them, a layer in one launch and in two
@pytest.mark.parametrize("m,n,k", [(1, 40_001, 700), (7, 600, 5000), (16, 300, 9000), (17, 30_003, 600), (31, 9000, 1500), (32, 70, 4000),
                                   (33, 4100, 300)])
def test_few_rows(m, n, k):
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(m + n + k)
    a, b = _whole(rng, m, k, 0), _whole(rng, n, k, 0)  # multiples of 1/4, at most 36 a product: exact up to 2^24 / 144 columns
    want = a.astype(np.float32) @ b.astype(np.float32).T
    out = torch.full((m + 1, n + 3), 7.0, dtype=torch.float32, device="cuda")
    sidco.sidco_mx4_matmul(*_upload(a), *_upload(b), k, out[:m, 1:n + 1])
    np.testing.assert_array_equal(_host(out[:m, 1:n + 1]), want)
    pb = _upload(b)
    layer = torch.full((m, n), 0.25, dtype=torch.float32, device="cuda")
    sidco.sidco_mx4_linear(_dev(a.astype(np.float32), "bfloat16"), *pb, layer, alpha=-2.0, accumulate=True)
    np.testing.assert_array_equal(_host(layer), 0.25 - 2.0 * want)
    out[:m, 1:n + 1] = 7.0
    assert bool((out == 7.0).all()), "written outside the result"


@pytest.mark.parametrize("m,n,k", [(1, 40, 300), (20, 40, 300), (200, 100, 600), (600, 600, 300)])
def test_blocks_that_stand_for_nan(m, n, k):
    """A row with such a block gives NaN in its whole row or column of the product and nowhere else."""
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(m)
    a, b = _whole(rng, m, k), _whole(rng, n, k)
    a[m // 2, k - 1] = np.nan
    b[3, 0] = np.inf
    out = torch.zeros((m, n), dtype=torch.float32, device="cuda")
    sidco.sidco_mx4_matmul(*_upload(a), *_upload(b), k, out)
    want = np.nan_to_num(ref.rounded(a)) @ np.nan_to_num(ref.rounded(b)).T
    want[m // 2, :] = np.nan
    want[:, 3] = np.nan
    np.testing.assert_array_equal(_host(out), want)


def test_training_products_against_differences():
    """The layer's gradients: with y = x^ W^^T, sum(y dy) changes by sum(dx_q e) when x^ moves by e, and likewise for W; the
    quantised output gradient is what both products see."""
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(3)
    rows, n, m = 70, 200, 130
    x, w, dy = _whole(rng, rows, n, 0), _whole(rng, m, n, 0), _whole(rng, rows, m, 0)
    forms = {}
    for name, t in (("x", x), ("w", w), ("dy", dy)):
        a, b = _packed(*t.shape), _packed(*t.shape[::-1])
        sidco.sidco_mx4_quantize(_dev(t.astype(np.float32)), *a, *b)
        forms[name] = a, b
    dx = torch.empty((rows, n), dtype=torch.float32, device="cuda")
    dw = torch.empty((m, n), dtype=torch.float32, device="cuda")
    sidco.sidco_mx4_matmul(*forms["dy"][0], *forms["w"][1], m, dx)
    sidco.sidco_mx4_matmul(*forms["dy"][1], *forms["x"][1], rows, dw)
    dyr, dyc, wc, xc = ref.rounded(dy), ref.rounded(dy.T).T, ref.rounded(w.T).T, ref.rounded(x.T).T
    np.testing.assert_array_equal(_host(dx), dyr @ wc)
    np.testing.assert_array_equal(_host(dw), dyc.T @ xc)
    e = rng.standard_normal((rows, n))
    h = 2.0 ** -10
    loss = lambda xx, ww, gg: float((xx @ ww.T * gg).sum())  # noqa: E731
    num = (loss(xc + h * e, wc, dyr) - loss(xc - h * e, wc, dyr)) / (2 * h)
    assert abs(num - float((_host(dx) * e).sum())) <= 1e-9 * np.abs(_host(dx) * e).sum() + 1e-6
    f = rng.standard_normal((m, n))
    num = (loss(xc, wc + h * f, dyc) - loss(xc, wc - h * f, dyc)) / (2 * h)
    assert abs(num - float((_host(dw) * f).sum())) <= 1e-9 * np.abs(_host(dw) * f).sum() + 1e-6


def test_streams_and_graph():
    """The layer's workspace belongs to the stream; a captured call replays on new inputs."""
    torch, sidco = _torch(), _sidco()
    rng = np.random.default_rng(4)
    rows, n, k = 24, 300, 800
    w = _upload(rng.standard_normal((n, k)))
    xs = [_dev(rng.standard_normal((rows, k)).astype(np.float32)) for _ in range(6)]
    want = []
    for x in xs:
        y = torch.empty((rows, n), dtype=torch.float32, device="cuda")
        sidco.sidco_mx4_linear(x, *w, y)
        want.append(_host(y))
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.empty((rows, n), dtype=torch.float32, device="cuda") for _ in xs]
    torch.cuda.synchronize()
    for i, x in enumerate(xs):
        with torch.cuda.stream(streams[i % 3]):
            sidco.sidco_mx4_linear(x, *w, outs[i])
    torch.cuda.synchronize()
    for o, e in zip(outs, want):
        np.testing.assert_array_equal(_host(o), e)
    x, y = xs[0].clone(), torch.empty((rows, n), dtype=torch.float32, device="cuda")
    side = streams[0]
    sidco.sidco_reserve(sidco.sidco_workspace_bytes_mx4_linear(rows, k), stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sidco.sidco_mx4_linear(x, *w, y, stream=side)
    for i in (1, 2, 3, 4):
        x.copy_(xs[i])
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(_host(y), want[i])
        _ = (xs[i] @ xs[i].t()).sum().item()


def test_binding_refuses():
    torch, sidco = _torch(), _sidco()
    x = torch.zeros((10, 300), device="cuda")
    a, b = _packed(10, 300), _packed(300, 10)
    with pytest.raises(TypeError):
        sidco.sidco_mx4_quantize(x.double(), *a)
    with pytest.raises(TypeError):
        sidco.sidco_mx4_quantize(x.t(), *b)
    with pytest.raises(TypeError):
        sidco.sidco_mx4_quantize(x.cpu(), *a)
    with pytest.raises(ValueError):
        sidco.sidco_mx4_quantize(x, a[0][:9], a[1])
    with pytest.raises(ValueError):
        sidco.sidco_mx4_quantize(x.expand(10, 300)[:1].expand(10, 300), *a)
    with pytest.raises(ValueError):
        sidco.sidco_mx4_matmul(*a, *a, 600, torch.zeros((10, 10), device="cuda"))
    with pytest.raises(ValueError):
        sidco.sidco_mx4_linear(x, *a, torch.zeros((9, 10), device="cuda"))
    with pytest.raises(ValueError):
        sidco.sidco_mx4_compress(x.view(-1), torch.zeros(100, device="cuda"), *_packed(1, 3000))
    with pytest.raises(ValueError):
        sidco.sidco_mx4_aggregate(*_packed(2, 256), torch.zeros(300, device="cuda"))
    with pytest.raises(sidco.SidcoError):
        sidco.sidco_mx4_quantize(x, None, None)
