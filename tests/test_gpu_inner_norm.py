"""The example with a norm in front: its weights stay as they are, so no gradient is formed that nobody uses."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from paper_2506_21263_amd import inner

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("base_bits", [8, 16])
def test_training_forms_no_gradient_of_the_norm(base_bits):
    dlcx.dlcx_profile_enable(True)
    try:
        inner.train(m=128, n=256, rows=32, inner=2, outer=1, base_bits=base_bits, norm=True)
        torch.cuda.synchronize()
        names = set(dlcx.dlcx_profile_read())
    finally:
        dlcx.dlcx_profile_enable(False)
    assert "rms_norm" in names and not names & {"rms_norm_backward", "rms_norm_sum"}
