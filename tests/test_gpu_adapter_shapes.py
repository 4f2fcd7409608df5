"""Factors, h and gradients in other layouts than the library's are refused, not read as if they had it."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV
from test_gpu_adapter import Case

pytestmark = pytest.mark.gpu


def test_factors_in_another_layout():
    c = Case(20, 64, 72, 8, 3, "bf16")
    y, h = c.out(c.y_in), torch.empty(c.rows, c.r, device=DEV)
    good = dict(d=c.d, x=c.x, ids=c.idd, q=c.qd, p=c.pd, y_in=c.y_in, y_out=y, h_out=h, workspace=c.workspace())
    turned = lambda t: t.transpose(-1, -2).contiguous()  # noqa: E731
    big = dict(q=torch.cat([c.pd, c.pd]), p=torch.cat([c.qd, c.qd]))  # enough elements, of the other side
    for bad in (dict(q=turned(c.qd)), dict(p=turned(c.pd)), big, dict(q=c.qd.view(8, 3, 72)), dict(h_out=turned(h)),
                dict(q=turned(c.qd.view(24, 72)))):
        with pytest.raises(ValueError):
            dlcx.dlcx_adapter_forward(**{**good, **bad})
    dx = c.out(c.dx_in)
    dq, dp = torch.empty(3, 8, 72, device=DEV), torch.empty(3, 8, 64, device=DEV)
    dlcx.dlcx_adapter_forward(**good)
    back = dict(d=c.d, x=c.x, dy=c.dy, ids=c.idd, q=c.qd, p=c.pd, h=h, dx_in=c.dx_in, dx_out=dx, dq_out=dq, dp_out=dp,
                workspace=c.workspace())
    for bad in (dict(q=turned(c.qd)), dict(h=turned(h)), dict(dq_out=turned(dq)), dict(dp_out=turned(dp)),
                dict(dp_out=dq)):
        with pytest.raises(ValueError):
            dlcx.dlcx_adapter_backward(**{**back, **bad})


def test_layouts_that_are_the_same_in_memory():
    c = Case(600, 64, 72, 8, 3, "f32", outside=False)
    y, h = c.forward()
    for q, p, hs in ((c.qd.view(-1), c.pd.view(-1), (c.rows * c.r,)), (c.qd.view(24, 72), c.pd.view(24, 64), (c.rows, c.r)),
                     (torch.cat([c.qd, c.qd]), torch.cat([c.pd, c.pd]), (c.rows + 5, c.r))):
        out, h2 = c.out(c.y_in), torch.empty(hs, device=DEV)
        dlcx.dlcx_adapter_forward(c.d, c.x, c.idd, q, p, c.y_in, out, h2, c.workspace(), scale=c.sd)
        assert torch.equal(out, y) and torch.equal(h2.view(-1)[:c.rows * c.r].view(c.rows, c.r), h)
