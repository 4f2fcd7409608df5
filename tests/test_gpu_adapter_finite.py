"""What is not finite in a row, a gradient or a factor goes where the formulas take it, and nowhere else."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV
from test_gpu_adapter import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,m,n,r,count", [(40, 136, 72, 12, 8), (300, 127, 130, 33, 4), (5000, 64, 264, 20, 3),
                                              (700, 264, 520, 70, 4)])
def test_columns_beyond_a_rank_are_zeros_whatever_the_rows_hold(rows, m, n, r, count, dtype):
    c = Case(rows, m, n, r, count, dtype, ranks=True, outside=False)
    assert 1 in c.rank and (count < 4 or 0 in c.rank)
    _, h = c.forward()
    for row, what in ((0, float("nan")), (rows // 2, float("inf")), (rows - 1, float("-inf"))):
        c.x[row, row % n] = what
        c.dy[row, row % m] = what
    for a in range(count):  # one more in a row of every adapter
        at = (c.ids == a).nonzero()[:, 0]
        if len(at):
            c.x[at[-1], n - 1] = float("nan")
            c.dy[at[-1], m - 1] = float("nan")
    _, dq, dp = c.backward(h)
    for a in range(count):
        assert not dq[a, c.rank[a]:].any() and not dp[a, c.rank[a]:].any(), a
        if c.rank[a] and (c.ids == a).any():
            assert torch.isnan(dq[a, 0]).any() and torch.isnan(dp[a, 0]).any(), a


def positive(rows, m, n, r, count, dtype, pad, ranks):
    """A case of positive numbers alone: sums of products in which an infinity stays one."""
    c = Case(rows, m, n, r, count, dtype, ranks=ranks, pad=pad, outside=False, seed=11)
    for name in ("x", "y_in", "dy", "dx_in"):
        t = getattr(c, name)
        t.copy_(t.abs() + 0.25)
    c.qd, c.pd = (t.abs().to(DEV) + 0.0625 for t in (c.q, c.p))
    return c


def formulas(c, h_in):
    """h, y, dx, dq, dp in 64 bits, adapter by adapter on the columns that there are."""
    x, y, dy, dx, s, h_in = (t.double().cpu() for t in (c.x, c.y_in, c.dy, c.dx_in, c.sd, h_in))
    q, p = c.qd.double().cpu(), c.pd.double().cpu()
    h, dq, dp = torch.zeros(c.rows, c.r).double(), torch.zeros(q.shape).double(), torch.zeros(p.shape).double()
    outer = lambda u, z: (u[:, :, None] * z[:, None, :]).sum(0)  # noqa: E731
    inner = lambda u, f: (u[:, None, :] * f[None]).sum(2)  # noqa: E731
    for a in range(c.count):
        at, k = (c.ids == a).nonzero()[:, 0], c.rank[a]
        if not len(at) or not k:
            continue
        ha = inner(x[at], q[a, :k])
        g = s[a] * inner(dy[at], p[a, :k])
        h[at, :k] = ha
        y[at] += s[a] * inner(ha, p[a, :k].t())
        dx[at] += inner(g, q[a, :k].t())
        dq[a, :k] = outer(g, x[at])
        dp[a, :k] = s[a] * outer(h_in[at, :k], dy[at])
    return h, y, dx, dq, dp


SIZES = [(7, 130, 67, 5, 2, 0), (70, 127, 509, 33, 2, 0), (201, 136, 72, 20, 3, 3), (90, 72, 136, 12, 4, 0),
         (333, 65, 1030, 70, 2, 0), (300, 520, 264, 40, 2, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,m,n,r,count,pad", SIZES)
@pytest.mark.parametrize("where", ["x", "dy", "q", "p", "h", "scale"])
def test_an_infinity_stays_one(where, rows, m, n, r, count, pad, dtype):
    c = positive(rows, m, n, r, count, dtype, pad, ranks=count > 3)
    _, h = c.forward()
    inf = float("inf")
    for a in range(count):  # the last of everything: what stands in for what is not there
        at, k = (c.ids == a).nonzero()[:, 0], c.rank[a]
        if not len(at) or not k:
            continue
        if where == "x":
            c.x[at[-1], n - 1] = c.x[at[0], n // 2] = inf
        elif where == "dy":
            c.dy[at[-1], m - 1] = c.dy[at[0], m // 2] = inf
        elif where == "q":
            c.qd[a, k - 1, n - 1] = inf
        elif where == "p":
            c.pd[a, k - 1, m - 1] = inf
        elif where == "h":
            h[at[-1], k - 1] = inf
        elif a == 0:
            c.sd[a] = inf
    want = formulas(c, h)
    y, h2 = c.forward()
    dx, dq, dp = c.backward(h)
    for name, got, v in zip(("h", "y", "dx", "dq", "dp"), (h2, y, dx, dq, dp), want):
        got = got.double().cpu()
        assert not torch.isnan(v).any() and torch.equal(torch.isinf(got), torch.isinf(v)), name
        assert not torch.isnan(got).any(), name
        # positive numbers: every sum is good to a few hundred roundings of 2^-24, and one of 2^-8
        fine = torch.isfinite(v)
        assert ((got - v).abs()[fine] <= (2.0 ** -8 + 2.0 ** -13) * v[fine]).all(), name
