"""GPU: cross entropy's gradient over several pieces of the vocabulary and its losses over several groups of rows where the operands are read
where they are, each gradient alone and on top of what is there."""
import pytest

import language_reference as ref
from test_gpu_cross_entropy import _case, _dtype, _near, _sidco, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("which,o,accumulate", [("both", "same", False), ("both", "f32", True), ("x", "same", False), ("w", "same", True), ("w", "f32", False)])
def test_pieces_of_operands_in_place(t, which, o, accumulate):
    torch, sidco = _torch(), _sidco()
    n, dim = 16_500, 64
    # words whose P both ways, in pairs but for bf16 gradients, are more than a piece of 2^30 bytes
    vocab = 2**30 // (n * 2 * (2 if which == "both" else 1) * (1 if t == "bf16" else 2)) + 1500
    o = t if o == "same" else o
    x, w, words = _case(n, dim, vocab, t, padding=0.3)
    g = torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    sidco.sidco_cross_entropy(x, w, words, loss, lse)
    dx = torch.full_like(x, 3.0) if which != "w" else None
    before = torch.randn(vocab, dim, device="cuda").mul_(0.1).to(_dtype(o)) if accumulate else None
    dw = None
    if which != "x":
        dw = before.clone() if accumulate else torch.full((vocab, dim), 3.0, dtype=_dtype(o), device="cuda")
    sidco.sidco_cross_entropy_grad(x, w, words, lse, g, dx, dw, accumulate=accumulate)
    torch.cuda.synchronize()
    r = ref.CrossEntropy(x, w, words, g)
    _near(lse, r.lse, r.lse_off, "lse")
    _near(loss, r.loss, r.loss_off, "loss")
    if dx is not None:
        _near(dx, *r.x_grad(), "x_grad")
    if dw is not None:
        _near(dw, *r.w_grad(_dtype(o), before), "w_grad")
