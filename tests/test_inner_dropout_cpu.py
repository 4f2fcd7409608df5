"""What a projection with dropout wants to know, on the host: nothing is launched."""
import pytest
import torch

from paper_2506_21263_amd import inner


def test_training_wants_the_number_of_the_step():
    proj = inner.AdapterProjection(torch.zeros(8, 8), torch.zeros(1, 2, 8), 1.0, 4, torch.float32, dropout=0.1)
    x = torch.zeros(4, 8)
    for call in (lambda: proj.forward(x, None), lambda: proj.backward(x, None, x, None)):
        with pytest.raises(ValueError, match="draw"):
            call()


def test_projections_have_seeds_of_their_own():
    make = lambda **kw: inner.AdapterProjection(torch.zeros(8, 8), torch.zeros(1, 2, 8), 1.0, 4, torch.float32, **kw)  # noqa: E731
    seeds = [make(dropout=0.1).seed for _ in range(3)]
    assert len(set(seeds)) == 3 and make(dropout=0.1, seed=seeds[0]).seed == seeds[0] and make(dropout=0.1, seed=0).seed == 0
