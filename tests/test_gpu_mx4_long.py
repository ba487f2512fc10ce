"""GPU: lengths whose blocks of threads are more than one dimension of a launch has room for (2^32 threads): against the same
numbers in pieces, bit for bit."""
import pytest

pytestmark = pytest.mark.gpu

PIECE = 1 << 27


def _torch():
    import torch
    return torch


def _sidco():
    import paper_2101_10761_amd as sidco
    return sidco


def _packed(rows, cols):
    torch, sidco = _torch(), _sidco()
    return (torch.full((sidco.sidco_mx4_code_bytes(rows, cols),), 0xA5, dtype=torch.uint8, device="cuda"),
            torch.full((sidco.sidco_mx4_scale_bytes(rows, cols),), 0xA5, dtype=torch.uint8, device="cuda"))


@pytest.fixture
def room():
    """These tests take up to 20 GB."""
    yield
    _torch().cuda.empty_cache()


@pytest.mark.parametrize("column", [False, True])
def test_a_vector_of_2_to_the_30(room, column):
    torch, sidco = _torch(), _sidco()
    n = (1 << 30) + 4711
    x = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    for at in range(0, n, PIECE):
        torch.randn(min(PIECE, n - at), dtype=torch.bfloat16, device="cuda", out=x[at:at + PIECE])

    def quantize(v, codes, scales):
        if column:
            sidco.sidco_mx4_quantize(v.view(-1, 1), None, None, codes, scales)
        else:
            sidco.sidco_mx4_quantize(v.view(1, -1), codes, scales)

    codes, scales = _packed(1, n)
    quantize(x, codes, scales)
    for at in range(0, n, PIECE):
        part = x[at:at + PIECE]
        c, s = _packed(1, part.numel())
        quantize(part, c, s)
        assert torch.equal(codes[at // 2:at // 2 + c.numel()], c) and torch.equal(scales[at // 32:at // 32 + s.numel()], s), at


def test_few_rows_by_2_to_the_27(room):
    torch, sidco = _torch(), _sidco()
    n, k = (1 << 27) + 1003, 32
    codes = torch.zeros((n, 128), dtype=torch.uint8, device="cuda")
    scales = torch.full((n, 8), 127, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for at in range(0, n, 1 << 24):
        rows = codes[at:at + (1 << 24), :16]
        rows.copy_(torch.randint(0, 256, rows.shape, dtype=torch.uint8, device="cuda", generator=g))
    x = torch.randint(-6, 7, (1, k), generator=torch.Generator().manual_seed(2)).float().cuda()
    x[0, 0] = 6.0  # whole numbers under one exponent: exact sums in any order
    a = _packed(1, k)
    sidco.sidco_mx4_quantize(x, *a)
    product, layer = torch.full((1, n), 7.0, device="cuda"), torch.full((1, n), 7.0, device="cuda")
    sidco.sidco_mx4_matmul(*a, codes, scales, k, product)
    sidco.sidco_mx4_linear(x, codes, scales, layer)
    assert torch.equal(product, layer)
    for at in range(0, n, 1 << 22):
        rows = min(1 << 22, n - at)
        want = torch.empty((1, rows), device="cuda")
        sidco.sidco_mx4_matmul(*a, codes[at:at + rows], scales[at:at + rows], k, want)
        assert torch.equal(product[:, at:at + rows], want), at
