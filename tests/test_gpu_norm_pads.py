"""The codes behind a row's end are zeros, whatever the row holds: a norm of NaN is NaN in the row's own elements alone."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from eight_ref import DEV, TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 5, 8, 130, 136, 513, 1000, 2050, 2056, 4100, 8195, 8200, 16392, 33001, 33000])
def test_codes_behind_a_row(n, dtype):
    x = torch.randn(4, n, device=DEV).to(TYPES[dtype])
    x[1, n // 2], x[3] = float("nan"), 0.0                 # rstd is NaN; and infinite, where eps is zero
    y8 = dlcx.fp8_empty(4, n, DEV)
    y8.held[0].view(torch.uint8).fill_(0x55)
    dlcx.dlcx_rms_norm(x, torch.ones(n, device=DEV, dtype=x.dtype), 0.0, y8_out=y8)
    codes = y8.held[0].view(torch.uint8)
    assert not bool(codes[:, n:].any())
    nan = (codes[:, :n] & 127) == 127
    assert bool(nan[[1, 3]].all()) and not bool(nan[[0, 2]].any())
