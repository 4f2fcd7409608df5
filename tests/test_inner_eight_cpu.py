"""What the projection with weights in 8 bits refuses, on the host."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from paper_2506_21263_amd import inner


def test_options_out_of_range():
    for bad in (dict(base_bits=4), dict(dropout=1.0), dict(dropout=-0.1), dict(dropout=float("nan"))):
        with pytest.raises(ValueError):
            inner.AdapterProjection(torch.zeros(8, 8), torch.zeros(1, 2, 8), 1.0, 4, torch.float32, **bad)


def test_tensors_of_the_wrong_kind():
    """What the binding refuses before an address is passed on (these live on the host)."""
    x, f16 = torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.float16)
    for call in (lambda: dlcx.dlcx_fp8_quantize(x), lambda: dlcx.dlcx_fp8_quantize(f16), lambda: dlcx.fp8(x, x, 8),
                 lambda: dlcx.fp8_empty(4, 8, "cpu"), lambda: dlcx.dlcx_rms_norm(x, x[0], 1e-5, y_out=x),
                 lambda: dlcx.dlcx_rms_norm(f16, f16[0], 1e-5, y_out=f16), lambda: dlcx.dlcx_dropout(x, None, x, 0.1, 1),
                 lambda: dlcx.dlcx_dropout(x, None, x, 0.1, -1), lambda: dlcx.dlcx_dropout(x, None, x, 0.1, 1, 1 << 64),
                 lambda: dlcx.dlcx_rms_norm_backward(x, x[0], x[:, 0], x, None, x, x[0], x)):
        with pytest.raises(ValueError):
            call()
