"""GPU: 4-bit products of sizes that take each of the tiles, in one launch and in two, with ragged edges: exact, so that every
element is compared.  Operands are multiples of 1/2 up to 6 under one exponent: products are multiples of 1/4 up to 36, and sums
of up to 2^24 / 144 of them are whole numbers of quarters that fp32 holds in any order.  test_dense_plans.py checks that these
sizes take the tiles that they are here for."""
import functools

import pytest

pytestmark = pytest.mark.gpu

# rows, columns, contraction: tiles of 64, 128, 192, 256; 256 and for the last columns 128, 64, 192
PRODUCTS = [(700, 601, 1500), (2100, 2050, 320), (2900, 2903, 4100), (3301, 3300, 4100), (4700, 4701, 4200), (5830, 5833, 2050), (4701, 4700, 9000)]
MODES = [("float32", 1.0, False), ("float32", -0.5, True), ("bfloat16", 1.0, False), ("float16", 0.25, True)]


def _torch():
    import torch
    return torch


def _sidco():
    import paper_2101_10761_amd as sidco
    return sidco


def _packed(rows, cols):
    torch, sidco = _torch(), _sidco()
    return (torch.empty(sidco.sidco_mx4_code_bytes(rows, cols), dtype=torch.uint8, device="cuda"),
            torch.empty(sidco.sidco_mx4_scale_bytes(rows, cols), dtype=torch.uint8, device="cuda"))


def _whole(rows, cols, seed):
    """A matrix that its blocks hold exactly, and the blocks."""
    torch, sidco = _torch(), _sidco()
    g = torch.Generator(device="cuda").manual_seed(seed)
    sizes = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device="cuda")
    x = sizes[torch.randint(0, 8, (rows, cols), generator=g, device="cuda")]
    x *= torch.randint(0, 2, (rows, cols), generator=g, device="cuda") * 2 - 1
    x[:, ::32] = 6.0  # the exponent of every block
    p, back = _packed(rows, cols), torch.empty_like(x)
    sidco.sidco_mx4_quantize(x, *p)
    sidco.sidco_mx4_dequantize(*p, back)
    assert torch.equal(x, back)
    return x, p


@functools.lru_cache(maxsize=1)
def _case(m, n, k):
    assert k <= 2 ** 24 // 144
    (a, pa), (b, pb) = _whole(m, k, m), _whole(n, k, n)
    return a, pa, b, pb, a @ b.t()


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype,alpha,accumulate", MODES)
def test_products(m, n, k, dtype, alpha, accumulate):
    torch, sidco = _torch(), _sidco()
    _, pa, _, pb, product = _case(m, n, k)
    buf = torch.full((m + 2, n + 3), 7.0, dtype=getattr(torch, dtype), device="cuda")
    out = buf[1:m + 1, 1:n + 1]
    old = torch.randint(-8, 9, (m, n), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(out.dtype)
    out.copy_(old)
    sidco.sidco_mx4_matmul(*pa, *pb, k, out, alpha=alpha, accumulate=accumulate)
    want = (alpha * product + (old.float() if accumulate else 0)).to(out.dtype)
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert bool((buf == 7.0).all()), "written outside the result"


@pytest.mark.parametrize("m,n,k", PRODUCTS[2:5])
def test_layers_on_many_rows(m, n, k):
    torch, sidco = _torch(), _sidco()
    a, _, _, pb, product = _case(m, n, k)
    x = torch.zeros((m, k + 5), dtype=torch.bfloat16, device="cuda")[:, 3:k + 3]
    x.copy_(a)
    out = torch.empty((m, n), device="cuda")
    sidco.sidco_mx4_linear(x, *pb, out)
    assert torch.equal(out, product)


@pytest.mark.parametrize("m,n,k", PRODUCTS[2:])
def test_blocks_that_stand_for_nan(m, n, k):
    """NaN in the row or column of such a block, in the first and the last tiles, and nowhere else."""
    torch, sidco = _torch(), _sidco()
    a, _, b, pb, product = _case(m, n, k)
    x = a.clone()
    x[0, k - 1] = float("nan")
    x[m - 1, 0] = float("inf")
    pa, out = _packed(m, k), torch.empty((m, n), device="cuda")
    sidco.sidco_mx4_quantize(x, *pa)
    sidco.sidco_mx4_matmul(*pa, *pb, k, out)
    assert bool(out[0].isnan().all()) and bool(out[m - 1].isnan().all())
    assert torch.equal(out[1:m - 1], product[1:m - 1])
