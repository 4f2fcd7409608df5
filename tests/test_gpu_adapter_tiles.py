"""Rows sorted into tiles: adapters with numbers of rows around the tiles' borders, beside matrices of any size.

All calls here have rows enough for that form (test_gpu_adapter_forms.py says which calls have)."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV
from test_gpu_adapter import Case, check
from test_gpu_adapter_finite import formulas, positive
from test_gpu_adapter_precision import inside, sharp

pytestmark = pytest.mark.gpu

SHARES = [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 256, 257, 300]  # rows of each adapter


def spread(c, shares, outside):
    """Gives the case's rows to adapters by these shares, in any order; the rest has none."""
    ids = torch.cat([torch.full((k,), a) for a, k in enumerate(shares)])
    rest = c.rows - len(ids)
    assert rest >= 0 and len(shares) == c.count
    ids = torch.cat([ids, torch.tensor([-1, c.count, -(1 << 31)])[torch.arange(rest) % 3]])
    if outside is not None:
        ids = ids[torch.randperm(c.rows, generator=torch.Generator().manual_seed(outside))]
    c.ids = ids.to(torch.int32)
    c.idd = c.ids.to(DEV)
    return c


def tiles_ran(call):
    dlcx.dlcx_profile_enable(True)
    out = call()
    torch.cuda.synchronize()
    names = dlcx.dlcx_profile_read()
    dlcx.dlcx_profile_enable(False)
    assert "adapter_up" in names and "adapter_rows" not in names, names
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,r,pad,shift", [(136, 72, 40, 0, 0), (127, 130, 33, 0, 0), (64, 65, 65, 0, 0), (72, 520, 100, 8, 0),
                                             (40, 24, 256, 0, 0), (33, 1030, 128, 3, 1), (7, 3, 64, 0, 0), (1, 1, 40, 0, 0),
                                             (520, 8, 48, 0, 0), (264, 2056, 32, 0, 0), (65, 4099, 17, 0, 0)])
def test_adapters_with_rows_around_the_borders(m, n, r, pad, shift, dtype):
    rows = sum(SHARES) + 40
    c = Case(rows, m, n, r, len(SHARES), dtype, ranks=r > 60, pad=pad, shift=shift, outside=False, seed=5)
    assert all((c.ids == a).any() for a in range(c.count))
    spread(c, SHARES, outside=m)
    y, h = tiles_ran(c.forward)
    tiles_ran(lambda: c.backward(h))
    check(c)


@pytest.mark.parametrize("rows,m,n,r,count", [(1300, 136, 520, 40, 3), (900, 264, 72, 64, 2), (700, 96, 264, 100, 3),
                                              (400, 264, 328, 256, 2), (1500, 127, 255, 33, 4), (3700, 65, 40, 3, 2)])
def test_y_and_dx_have_one_rounding_in_tiles(rows, m, n, r, count):
    c = Case(rows, m, n, r, count, "bf16", ranks=count > 2)
    c.dy = (c.dy * 8).contiguous()
    want_y, want_dx = sharp(c)
    y, h = tiles_ran(lambda: c.forward(y_in=None))
    inside(y, want_y, "y")
    dx = torch.empty(rows, n, device=DEV, dtype=torch.bfloat16)
    dq, dp = (torch.empty(count, r, k, device=DEV) for k in (n, m))
    tiles_ran(lambda: dlcx.dlcx_adapter_backward(c.d, c.x, c.dy, c.idd, c.qd, c.pd, h, None, dx, dq, dp, c.workspace(),
                                                 scale=c.sd, ranks=c.ranks))
    inside(dx, want_dx, "dx")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,r,pad", [(130, 67, 45, 0), (127, 509, 33, 0), (136, 72, 70, 3), (65, 1030, 130, 0), (264, 136, 40, 8)])
@pytest.mark.parametrize("where", ["x", "dy", "q", "p", "h", "scale"])
def test_an_infinity_stays_one_in_tiles(where, m, n, r, pad, dtype):
    shares = [1, 17, 33, 79, 300, 900]
    c = positive(sum(shares), m, n, r, len(shares), dtype, pad, ranks=False)
    spread(c, shares, outside=r)
    _, h = c.forward()
    inf = float("inf")
    for a in range(c.count):
        at, k = (c.ids == a).nonzero()[:, 0], c.rank[a]
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
        elif a == 4:
            c.sd[a] = inf
    want = formulas(c, h)
    y, h2 = tiles_ran(c.forward)
    dx, dq, dp = tiles_ran(lambda: c.backward(h))
    for name, got, v in zip(("h", "y", "dx", "dq", "dp"), (h2, y, dx, dq, dp), want):
        got = got.double().cpu()
        assert not torch.isnan(v).any() and torch.equal(torch.isinf(got), torch.isinf(v)), name
        assert not torch.isnan(got).any(), name
        fine = torch.isfinite(v)
        assert ((got - v).abs()[fine] <= (2.0 ** -8 + 2.0 ** -13) * v[fine]).all(), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_updates_in_place_in_tiles(dtype):
    c = Case(2000, 136, 72, 24, 3, dtype)
    y, h = tiles_ran(c.forward)
    place = c.y_in.clone()
    tiles_ran(lambda: c.forward(y_in=place, y_out=place))
    assert torch.equal(place, y)
    dx = c.dx_in.clone()
    dq, dp = (torch.empty(c.count, c.r, k, device=DEV) for k in (c.n, c.m))
    dlcx.dlcx_adapter_backward(c.d, c.x, c.dy, c.idd, c.qd, c.pd, h, dx, dx, dq, dp, c.workspace(), scale=c.sd)
    for got, one in zip((dx, dq, dp), c.backward(h)):
        assert torch.equal(got, one)
    y, _ = tiles_ran(lambda: c.forward(y_in=torch.zeros_like(c.y_in)))
    z, _ = c.forward(y_in=None)
    assert torch.equal(y, z)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1600, 5000])
def test_values_that_are_not_finite_stay_in_their_rows_in_tiles(rows, dtype):
    c, clean = (Case(rows, 128, 128, 48, 3, dtype) for _ in range(2))
    c.x[3, 5] = float("nan")
    c.x[7, 1] = float("inf")
    c.y_in[11, 2] = float("-inf")
    lost = torch.zeros(rows, dtype=torch.bool)
    lost[[3, 7]] = True
    lost &= (c.ids >= 0) & (c.ids < c.count)
    y, _ = tiles_ran(c.forward)
    y2, _ = clean.forward()
    keep = ~lost
    keep[11] = False
    assert torch.equal(y[keep.to(DEV)], y2[keep.to(DEV)]) and y[11, 2] == float("-inf")
    assert not torch.isfinite(y[lost.to(DEV)]).all(1).any()
