"""Matrices in 8 bits whose scales are NaN (a byte of 255), in every form of the product and in the decoder."""
import numpy as np
import pytest
import torch

import paper_2506_21263_amd as dlcx
from eight_ref import DEV, HALF, TYPES, f64
from test_gpu_fp8 import operand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,m", [(1, 90), (16, 5000), (20, 90), (100, 300), (128, 40), (300, 130), (700, 700), (2048, 1024), (4096, 2048)])
def test_a_scale_that_is_nan(rows, m, dtype, zeros):
    """A byte of 255 in one row of x and one of w, beside other scales below 1: all outputs of that row and of that column
    are NaN, of zeros too, and no other is."""
    n = 700                                            # six blocks, the last one in the second quad of scales
    gen = torch.Generator().manual_seed(rows + m)
    x, xv = operand(gen, rows, n)
    w, wv = operand(gen, m, n)
    for a, row, block in ((x, rows - 1, 5), (w, 7, 1)):
        a.held[1][row, block] = 255
        if zeros:
            a.held[0].view(torch.uint8)[row, block * 128:block * 128 + 128] = 0
    y = torch.empty(rows, m, device=DEV, dtype=TYPES[dtype])
    ws = torch.empty(dlcx.dlcx_fp8_product_workspace_bytes(rows, m, n), device=DEV, dtype=torch.uint8)
    dlcx.dlcx_fp8_product(x, w, None, y, ws)
    bad = torch.zeros(rows, m, dtype=torch.bool)
    bad[rows - 1], bad[:, 7] = True, True
    assert torch.equal(y.isnan().cpu(), bad)
    if rows > 1:
        ok, most = ~bad.numpy(), np.abs(xv) @ np.abs(wv).T
        bound = ((n + 8) * 2.0 ** -23 + (2.0 ** -10 + HALF[y.dtype] * 1.01 if dtype == "bf16" else 0)) * most
        assert (np.abs(f64(y) - xv @ wv.T) <= bound)[ok].all()


def test_a_scale_that_is_nan_is_decoded_as_one():
    gen = torch.Generator().manual_seed(7)
    a, v = operand(gen, 5, 300)
    a.held[1][3, 1] = 255
    a.held[0].view(torch.uint8)[3, 130] = 0
    bad = np.zeros((5, 300), bool)
    bad[3, 128:256] = True
    for dt in TYPES.values():
        out = torch.empty(5, 300, device=DEV, dtype=dt)
        dlcx.dlcx_fp8_decode(a, out)
        assert np.array_equal(np.isnan(f64(out)), bad) and np.array_equal(f64(out)[~bad], v[~bad])
