"""Adapters whose launches have more than 2^32 threads: 512 of rank 1 beside 2^24 outputs (34 GB of factors)."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV

pytestmark = pytest.mark.gpu


def test_more_workgroups_than_a_launch_has_along_x():
    rows, m, n, count = 520, 1 << 24, 8, 512
    d = dlcx.adapter_desc(m, n, 1, count, dlcx.F32)
    z = lambda *s, t=torch.float32: torch.zeros(*s, device=DEV, dtype=t)  # noqa: E731
    ids = (torch.arange(rows, device=DEV) * 7 % count).to(torch.int32)
    at = torch.tensor([0, 1, 63, 64, (1 << 23) + 5, m - 65, m - 1], device=DEV)
    x, q, p = z(rows, n), z(count, 1, n), z(count, 1, m)
    x[:, 3], q[:, 0, 3] = 2.0, 0.5                                # h = 1
    value = 1.0 + torch.arange(count, device=DEV)
    p[:, 0, at] = value[:, None]
    y, h = z(rows, m), z(rows, 1)
    y.fill_(float("nan"))
    ws = z(dlcx.dlcx_adapter_workspace_bytes(d, rows), t=torch.uint8)
    dlcx.dlcx_adapter_forward(d, x, ids, q, p, None, y, h, ws)
    assert (h == 1).all() and torch.equal(y[:, at], value[ids.long()][:, None].expand(-1, len(at)))
    assert int(y.count_nonzero()) == rows * len(at) and not torch.isnan(y).any()
    # g = sum over the seven columns of y p = 7 value^2, dP = sum over an adapter's rows of y
    dx, dq, dp = z(rows, n), z(count, 1, n), z(count, 1, m)
    dp.fill_(float("nan"))
    dlcx.dlcx_adapter_backward(d, x, y, ids, q, p, h, None, dx, dq, dp, ws)
    g = 7.0 * value[ids.long()] ** 2                              # whole numbers below 2^24
    assert torch.equal(dx[:, 3], 0.5 * g) and int(dx.count_nonzero()) == rows
    times = torch.bincount(ids.long(), minlength=count).float()
    assert torch.equal(dq[:, 0, 3], 2.0 * 7.0 * value ** 2 * times)
    assert torch.equal(dp[:, 0, at], (value * times)[:, None].expand(-1, len(at)))
    assert int(dp.count_nonzero()) == int((times > 0).sum()) * len(at) and not torch.isnan(dp).any()
