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
