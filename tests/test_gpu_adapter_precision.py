"""bf16 adapters carry h and g in all their 32 bits: a row's result does not hang on how many others share its call.

Bounds: u = 2^-24 for every operation of an fp32 sum (its length and a few more, times the sum of magnitudes), 2^-32 for
a piece of h that stands for a zero, and one rounding of the result to bf16 (2^-8).  A single rounding of h to bf16
would add 2^-8 of the magnitudes that cancel in the second product."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV
from test_gpu_adapter import BF, U, Case, inside

pytestmark = pytest.mark.gpu


def sharp(c):
    """y - y_in and dx - dx_in in 64 bits, and bounds without a rounding of h or g."""
    d = {k: getattr(c, k).double().cpu() for k in ("x", "dy", "scale")}
    y, ey = torch.zeros(c.rows, c.m).double(), torch.zeros(c.rows, c.m).double()
    dx, ex = torch.zeros(c.rows, c.n).double(), torch.zeros(c.rows, c.n).double()
    for a in range(c.count):
        at, k, s = (c.ids == a).nonzero()[:, 0], c.rank[a], d["scale"][a]
        if not len(at) or not k:
            continue
        q, p = c.q[a, :k].double(), c.p[a, :k].double()
        for src, first, second, length, out, err in ((d["x"], q, p, c.n, y, ey), (d["dy"], p, q, c.m, dx, ex)):
            h = s * (src[at] @ first.t())
            eh = s * (length + 16) * U * (src[at].abs() @ first.abs().t())
            out[at] = h @ second
            # three products of pieces instead of one, so three times the additions
            err[at] = (eh + (3 * (c.r + 16) + 2) * U * h.abs()) @ second.abs()
    return (y, ey + BF * (y.abs() + ey)), (dx, ex + BF * (dx.abs() + ex))


@pytest.mark.parametrize("rows,m,n,r,count", [(300, 136, 520, 20, 3), (513, 264, 72, 64, 2), (150, 96, 264, 100, 3),
                                              (70, 264, 328, 256, 2), (400, 127, 255, 33, 4)])
def test_y_and_dx_have_one_rounding(rows, m, n, r, count):
    c = Case(rows, m, n, r, count, "bf16", ranks=count > 2)
    c.dy = (c.dy * 8).contiguous()
    want_y, want_dx = sharp(c)
    y, h = c.forward(y_in=None)
    inside(y, want_y, "y")
    dx = torch.empty(rows, n, device=DEV, dtype=torch.bfloat16)
    dq, dp = (torch.empty(count, r, k, device=DEV) for k in (n, m))
    dlcx.dlcx_adapter_backward(c.d, c.x, c.dy, c.idd, c.qd, c.pd, h, None, dx, dq, dp, c.workspace(), scale=c.sd,
                               ranks=c.ranks)
    inside(dx, want_dx, "dx")


def test_what_cancels_in_the_second_product():
    # two columns of h of 1 + 2^-9 and -1: bf16 has no room for the first, and the rest is all that y is
    rows, n, m = 3000, 16, 64
    c = Case(rows, m, n, 2, 1, "bf16", order="one")
    c.x = torch.zeros(rows, n, device=DEV, dtype=torch.bfloat16)
    c.x[:, 0], c.x[:, 1] = 1.0, 2.0 ** -9
    c.qd = torch.zeros(1, 2, n, device=DEV, dtype=torch.bfloat16)
    c.qd[0, 0, 0], c.qd[0, 0, 1], c.qd[0, 1, 0] = 1.0, 1.0, -1.0
    c.pd = torch.ones(1, 2, m, device=DEV, dtype=torch.bfloat16)
    c.sd = torch.ones(1, device=DEV)
    y, h = c.forward(y_in=None)
    assert (h[:, 0] == 1 + 2.0 ** -9).all() and (y == 2.0 ** -9).all()


def test_an_infinity_times_any_number_is_that_infinity():
    """Pieces of a number have its sign and none is zero: h times an infinite element of the factor does not become NaN."""
    rows, n, m = 2100, 32, 72
    c = Case(rows, m, n, 2, 1, "bf16", order="one")
    value = torch.tensor([1.0, -3.0, 1.0 + 2.0 ** -7, 2.0 ** -60, -(2.0 ** 100), 0.3, 256.5], dtype=torch.float32)
    c.x = torch.zeros(rows, n, device=DEV, dtype=torch.bfloat16)
    c.x[:, 0] = value[torch.arange(rows) % len(value)].to(torch.bfloat16).to(DEV)
    c.qd = torch.zeros(1, 2, n, device=DEV, dtype=torch.bfloat16)
    c.qd[0, 0, 0], c.qd[0, 1, 0] = 1.0, 1.0
    c.pd = torch.ones(1, 2, m, device=DEV, dtype=torch.bfloat16)
    c.pd[0, 0, 5], c.pd[0, 0, 6] = float("inf"), float("-inf")
    c.sd = torch.ones(1, device=DEV)
    y, _ = c.forward(y_in=None)
    sign = torch.sign(c.x[:, 0]).float()
    assert torch.equal(y[:, 5].float(), sign * float("inf")) and torch.equal(y[:, 6].float(), -sign * float("inf"))
    keep = [j for j in range(m) if j not in (5, 6)]
    assert torch.isfinite(y[:, keep]).all()
    # and an infinite h: every column of the row is infinite, of the factor's sign
    c.pd = torch.ones(1, 2, m, device=DEV, dtype=torch.bfloat16)
    c.pd[0, :, 1::2] = -1.0
    c.x[7, 0] = float("inf")
    y, _ = c.forward(y_in=None)
    assert (y[7, 0::2] == float("inf")).all() and (y[7, 1::2] == float("-inf")).all()
