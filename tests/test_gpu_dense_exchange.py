"""GPU: the exchanges of the training run say what they send: the sparse one the pairs that were selected, not the ratio's target."""
import pytest

pytestmark = pytest.mark.gpu


def test_bytes_are_those_of_the_pairs_selected():
    import torch
    from paper_2101_10761_amd import dense_step
    d, delta, workers = 100_000, 0.05, 2
    swap = dense_step.ExchangeSparse(workers, d, torch.device("cuda"), delta)
    selected = []
    for step in range(3):
        for w in range(workers):
            g = torch.randn(d, generator=torch.Generator(device="cuda").manual_seed(10 * step + w), device="cuda") * 1e-3
            swap.send(w, g)
            selected.append(int(swap.count[w]))
    assert swap.bytes == 8 * sum(selected) / len(selected)
    assert swap.bytes != 8 * delta * d  # normal numbers are not the law's: their count is off the target
    dense = dense_step.Exchange4Bit(workers, d, torch.device("cuda"))
    assert dense.bytes == dense.codes[0].numel() + dense.scales[0].numel()
