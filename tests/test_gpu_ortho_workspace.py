"""GPU: the bytes that the host helper gives for a call are enough for it, whatever its steps, coefficients and precision."""
import pytest

from test_gpu_ortho import _sidco, _torch

pytestmark = pytest.mark.gpu

USUAL = (3.4445, -4.7750, 2.0315)


@pytest.mark.parametrize("steps,coef", [(1, USUAL), (2, USUAL), (5, USUAL), (7, USUAL), (11, USUAL), (5, (4.5, -8.4, 3.5)), (3, (1.5, -0.5, 0.0))])
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("precision", [0, 1, 2])
def test_a_workspace_of_the_helpers_size(steps, coef, dtype, precision):
    torch, sidco = _torch(), _sidco()
    batch, rows, cols = 2, 200, 900
    x = torch.randn(batch, rows, cols, generator=torch.Generator(device="cuda").manual_seed(steps), device="cuda")
    want, out = (torch.empty(x.shape, dtype=getattr(torch, dtype), device="cuda") for _ in range(2))
    sidco.sidco_orthogonalize(x, want, steps=steps, coef=coef, precision=precision)
    code = {"float32": sidco.GRAD_F32, "float16": sidco.GRAD_F16, "bfloat16": sidco.GRAD_BF16}[dtype]
    need = sidco.sidco_workspace_bytes_orthogonalize(batch, rows, cols, code, precision, steps, coef)
    buf = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    try:
        sidco.sidco_set_workspace(buf[:need])
        sidco.sidco_orthogonalize(x, out, steps=steps, coef=coef, precision=precision)
    finally:
        torch.cuda.synchronize()
        sidco.sidco_set_workspace(None)
    assert torch.equal(out, want)
    assert bool((buf[need:] == 0x5A).all()), "written past the workspace"
