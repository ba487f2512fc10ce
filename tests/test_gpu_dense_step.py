"""GPU: the dense operators together in a training run, with the 4-bit and with the sparse exchange."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exchange", ["4bit", "sparse"])
def test_training_learns_and_answers(exchange):
    from paper_2101_10761_amd import dense_step
    r = dense_step.train(exchange, workers=2, steps=30, batch=128, sizes=(96, 160, 40))
    first, last = r["losses"][0], sum(r["losses"][-3:]) / 3
    assert last < 0.7 * first, r["losses"]
    # a row alone and among others: the same products with sums in another order, which may move a code of the layer between
    assert r["answers"][0] <= 0.05 * r["answers"][1]
    assert r["bytes"] < r["gradient_bytes"] / 2
