"""Low-rank adapters beside a shared projection and their gradient, against the formulas in 64 bits.

Bounds are those of the arithmetic, element by element: u = 2^-24 per addition of an fp32 sum (its length
plus a few, times the sum of magnitudes), 2^-8 for a value rounded to bf16 (8 significant bits), 2^-24 for one
in three bf16 pieces; fp32 forms have the u terms alone."""
import numpy as np
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = 2.0 ** -8
PIECES = 2.0 ** -24


class Case:
    def __init__(self, rows, m, n, r, count, dtype, order="mixed", ranks=False, seed=0, pad=0, shift=0,
                 outside=True):
        self.rows, self.m, self.n, self.r, self.count = rows, m, n, r, count
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.d = dlcx.adapter_desc(m, n, r, count, dlcx.BF16 if dtype == "bf16" else dlcx.F32)
        gen = torch.Generator().manual_seed(seed + 7 * rows + r)
        rnd = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)  # noqa: E731

        def matrix(cols, std=1.0):
            """A view of `rows` rows inside a larger array whose other elements are NaN."""
            full = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=self.dt)
            view = full[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
            view.copy_((rnd(rows, cols) * std).to(self.dt))
            full = full.to(DEV)
            return full[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]

        self.x, self.y_in, self.dy, self.dx_in = matrix(n), matrix(m), matrix(m, 0.01), matrix(n, 0.01)
        self.q = (rnd(count, r, n) * 0.1).to(self.dt)
        self.p = (rnd(count, r, m) * 0.1).to(self.dt)
        self.scale = (torch.rand(count, generator=gen) + 0.5).float()
        if order == "mixed":
            self.ids = torch.randint(-1 if outside else 0, count + (1 if outside else 0), (rows,), generator=gen)
        elif order == "none":
            self.ids = torch.full((rows,), -1)
        elif order == "one":
            self.ids = torch.full((rows,), count - 1)
        else:
            self.ids = torch.arange(rows) * count // rows
        self.ids = self.ids.to(torch.int32)
        self.ranks = None
        self.rank = [r] * count
        if ranks:
            self.rank = [[r, (r + 1) // 2, 1, 0][a % 4] for a in range(count)]
            self.ranks = torch.tensor(self.rank, dtype=torch.int32, device=DEV)
        for a in range(count):  # what is not to be read
            used = bool((self.ids == a).any())
            self.q[a, self.rank[a] if used else 0:] = float("nan")
            self.p[a, self.rank[a] if used else 0:] = float("nan")
        self.qd, self.pd, self.sd, self.idd = (t.to(DEV) for t in (self.q, self.p, self.scale, self.ids))

    def oracle(self):
        """Values and bounds of h, y, dx, dq, dp."""
        d = {k: getattr(self, k).double().cpu() for k in ("x", "y_in", "dy", "dx_in", "scale")}
        q, p = self.q.double(), self.p.double()
        low = self.dt == torch.bfloat16
        r = self.r
        h, eh = torch.zeros(self.rows, r).double(), torch.zeros(self.rows, r).double()
        y, ey = d["y_in"].clone(), torch.zeros_like(d["y_in"])
        dx, ex = d["dx_in"].clone(), torch.zeros_like(d["dx_in"])
        dq, dp = torch.zeros(q.shape).double(), torch.zeros(p.shape).double()
        eq, ep = dq.clone(), dp.clone()
        for a in range(self.count):
            at, k, s = (self.ids == a).nonzero()[:, 0], self.rank[a], d["scale"][a]
            if not len(at) or not k:
                continue
            x, dy, qa, pa = d["x"][at], d["dy"][at], q[a, :k], p[a, :k]
            ha = x @ qa.t()
            eha = (self.n + 16) * U * (x.abs() @ qa.abs().t())
            h[at, :k], eh[at, :k] = ha, eha
            y[at] += s * (ha @ pa)
            ey[at] = s * ((eha + ((r + 16) * U + (BF if low else 0)) * ha.abs()) @ pa.abs())
            g = s * (dy @ pa.t())
            eg = s * (self.m + 17) * U * (dy.abs() @ pa.abs().t())
            dx[at] += g @ qa
            ex[at] = (eg + ((r + 16) * U + (BF if low else 0)) * g.abs()) @ qa.abs()
            # (the gradient of P takes h as the forward call left it)
            piece = (PIECES if low else 0) + (len(at) + 16) * U
            dq[a, :k] = g.t() @ x
            eq[a, :k] = (eg + piece * g.abs()).t() @ x.abs()
            dp[a, :k] = s * (ha.t() @ dy)
            ep[a, :k] = s * ((eha + piece * ha.abs()).t() @ dy.abs())
        last = BF if low else 2 * U
        return {"h": (h, eh), "y": (y, ey + last * (y.abs() + ey)), "dx": (dx, ex + last * (dx.abs() + ex)),
                "dq": (dq, eq + U * dq.abs()), "dp": (dp, ep + U * dp.abs())}

    def workspace(self, rows=None):
        n = dlcx.dlcx_adapter_workspace_bytes(self.d, self.rows if rows is None else rows)
        return torch.full((n,), 0xFF, device=DEV, dtype=torch.uint8)

    def out(self, like):
        """An output of the same strides, all NaN."""
        return torch.full_like(like, float("nan")) if like.is_contiguous() else torch.empty_strided(
            like.shape, like.stride(), dtype=like.dtype, device=DEV).fill_(float("nan"))

    def forward(self, route=None, y_in="given", ws=None, y_out=None, h=None):
        y = self.out(self.y_in) if y_out is None else y_out
        h = torch.full((self.rows, self.r), float("nan"), device=DEV) if h is None else h
        dlcx.dlcx_adapter_forward(self.d, self.x, self.idd, self.qd, self.pd,
                                  self.y_in if isinstance(y_in, str) else y_in, y, h,
                                  self.workspace() if ws is None else ws, scale=self.sd, ranks=self.ranks, route=route)
        return y, h

    def backward(self, h, route=None, ws=None):
        dx = self.out(self.dx_in)
        dq = torch.full((self.count, self.r, self.n), float("nan"), device=DEV)
        dp = torch.full((self.count, self.r, self.m), float("nan"), device=DEV)
        dlcx.dlcx_adapter_backward(self.d, self.x, self.dy, self.idd, self.qd, self.pd, h, self.dx_in, dx, dq, dp,
                                   self.workspace() if ws is None else ws, scale=self.sd, ranks=self.ranks, route=route)
        return dx, dq, dp


def inside(got, want, name):
    value, bound = want
    off = (got.double().cpu() - value).abs()
    assert torch.isfinite(off).all(), name
    bad = off > bound + 1e-30
    assert not bad.any(), (name, int(bad.sum()), bad.nonzero()[:3].tolist(), float((off / (bound + 1e-30)).max()))


def check(c):
    want = c.oracle()
    y, h = c.forward()
    inside(h, want["h"], "h")
    inside(y, want["y"], "y")
    dx, dq, dp = c.backward(h)
    for name, got in (("dx", dx), ("dq", dq), ("dp", dp)):
        inside(got, want[name], name)


CASES = [
    # the smallest sizes, and one row
    dict(rows=1, m=1, n=1, r=1, count=1, order="one"), dict(rows=1, m=2048, n=2048, r=8, count=4, outside=False),
    dict(rows=2, m=7, n=3, r=3, count=2), dict(rows=3, m=16, n=600, r=5, count=1, order="one"),
    # around the tiles' borders: 16, 64, 256 rows; 64 and 128 columns; 32 columns of a factor
    dict(rows=15, m=128, n=64, r=16, count=1, order="one"), dict(rows=16, m=130, n=66, r=17, count=2),
    dict(rows=17, m=64, n=128, r=31, count=3), dict(rows=63, m=136, n=520, r=32, count=1, order="one"),
    dict(rows=64, m=256, n=1032, r=33, count=1, order="one"), dict(rows=65, m=65, n=129, r=64, count=2),
    dict(rows=257, m=127, n=255, r=65, count=4), dict(rows=130, m=96, n=512, r=100, count=2, ranks=True),
    # the largest rank; many adapters; ranks of zero
    dict(rows=70, m=264, n=328, r=256, count=3), dict(rows=90, m=64, n=64, r=4, count=300, ranks=True),
    dict(rows=40, m=24, n=40, r=8, count=1024), dict(rows=33, m=40, n=24, r=12, count=8, ranks=True),
    # nobody has an adapter
    dict(rows=50, m=72, n=80, r=8, count=3, order="none"),
    # rows of 16 bytes and rows that are not, views with a stride, first elements off 16 bytes
    dict(rows=100, m=1021, n=509, r=20, count=3), dict(rows=77, m=128, n=192, r=24, count=2, pad=8),
    dict(rows=77, m=128, n=192, r=24, count=2, pad=3), dict(rows=31, m=64, n=64, r=8, count=2, shift=1),
    # enough rows for tiles of 64 in the down product, of 256 and more in the others, and for several of an adapter
    dict(rows=4099, m=512, n=264, r=40, count=3, order="equal"), dict(rows=2500, m=96, n=2048, r=128, count=2),
    dict(rows=9001, m=40, n=72, r=12, count=2), dict(rows=20000, m=16, n=16, r=2, count=5),
    dict(rows=16500, m=2080, n=72, r=16, count=1, order="one"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join("%s" % v for v in c.values()))
def test_adapters_and_their_gradient_against_64_bits(case, dtype):
    check(Case(dtype=dtype, **case))


FEW = [(1, 2048, 2048, 8, 3), (1, 1, 1, 1, 1), (3, 5, 7, 2, 2), (2, 7, 1000, 5, 4), (2, 1025, 513, 17, 9), (40, 1023, 8, 100, 5),
       (7, 1030, 2049, 33, 2), (1, 512, 4097, 16, 1), (9, 2047, 515, 256, 3),  # one launch
       (5, 4096, 8192, 64, 4), (600, 333, 65, 6, 64), (20, 4101, 8191, 8, 7)]  # two (the last: in fp32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,m,n,r,count", FEW)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
def test_few_rows_at_the_edges_of_their_forms(rows, m, n, r, count, dtype, pad, shift):
    c = Case(rows, m, n, r, count, dtype, ranks=count > 2, seed=m, pad=pad, shift=shift)
    want = c.oracle()
    y, h = c.forward()
    inside(h, want["h"], "h")
    inside(y, want["y"], "y")


@pytest.mark.parametrize("dtype,rows", [("bf16", 1600), ("f32", 800)])
@pytest.mark.parametrize("m,n,r", [(264, 8200, 20), (8200, 264, 64), (7752, 7752, 9)])
def test_matrices_that_are_streamed(dtype, rows, m, n, r):
    check(Case(rows, m, n, r, 3, dtype, ranks=r == 64, seed=2, pad=8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_routes_and_workspaces_serve_what_they_promise(dtype):
    c = Case(700, 264, 520, 24, 6, dtype, ranks=True)
    ws = c.workspace()
    y, h = c.forward(ws=ws)
    grads = c.backward(h, ws=ws)
    route = torch.empty(dlcx.dlcx_adapter_route_bytes(c.rows, c.count), device=DEV, dtype=torch.uint8)
    dlcx.dlcx_adapter_route(c.idd, c.count, route)
    big = c.workspace(5000)  # room for more rows has room for fewer
    y2, h2 = c.forward(route=route, ws=big)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    for a, b in zip(grads, c.backward(h, route=route, ws=big)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 300])
def test_zeros_and_updates_in_place(dtype, rows):
    c = Case(rows, 136, 72, 12, 3, dtype)
    want = c.oracle()
    value, bound = want["y"]
    base = c.y_in.double().cpu()
    y, _ = c.forward(y_in=None)
    low = BF if dtype == "bf16" else 2 * U
    inside(y, (value - base, bound + low * (value - base).abs()), "y without y_in")
    y, h = c.forward()
    place = c.y_in.clone()
    c.forward(y_in=place, y_out=place)
    assert torch.equal(place, y)
    dx = c.dx_in.clone()
    dq, dp = (torch.empty(c.count, c.r, k, device=DEV) for k in (c.n, c.m))
    dlcx.dlcx_adapter_backward(c.d, c.x, c.dy, c.idd, c.qd, c.pd, h, dx, dx, dq, dp, c.workspace(), scale=c.sd)
    for got, one in zip((dx, dq, dp), c.backward(h)):
        assert torch.equal(got, one)


def test_no_scale_means_one():
    c = Case(40, 64, 64, 8, 2, "f32", outside=False)
    c.scale.fill_(1.0)
    want = c.oracle()
    y, h = c.out(c.y_in), torch.empty(c.rows, c.r, device=DEV)
    dlcx.dlcx_adapter_forward(c.d, c.x, c.idd, c.qd, c.pd, c.y_in, y, h, c.workspace())
    inside(y, want["y"], "y")


def test_rows_without_an_adapter_keep_what_is_not_finite_to_themselves():
    for dtype in ("bf16", "f32"):
        c = Case(200, 128, 128, 16, 3, dtype)
        c.x[3, 5] = float("nan")
        c.x[7, 1] = float("inf")
        c.y_in[11, 2] = float("-inf")
        lost = torch.zeros(c.rows, dtype=torch.bool)
        lost[[3, 7]] = True
        lost &= (c.ids >= 0) & (c.ids < c.count)
        y, _ = c.forward()
        clean = Case(200, 128, 128, 16, 3, dtype)
        y2, _ = clean.forward()
        keep = ~lost
        keep[11] = False
        assert torch.equal(y[keep.to(DEV)], y2[keep.to(DEV)])
        assert y[11, 2] == float("-inf")
        assert not torch.isfinite(y[lost.to(DEV)]).all(1).any()


def test_a_gradient_is_the_difference_of_the_loss():
    # y is linear in Q and in P, so a central difference has no error of its own at any step
    c = Case(150, 72, 88, 10, 3, "f32", outside=False)
    w = torch.randn(c.rows, c.m, generator=torch.Generator().manual_seed(1)).to(DEV)
    c.dy = w
    _, h = c.forward()
    _, dq, dp = c.backward(h)
    for name, grad in (("qd", dq), ("pd", dp)):
        old = getattr(c, name)
        step = torch.randn(old.shape, generator=torch.Generator().manual_seed(2)).to(DEV) * 0.1
        loss = []
        for sign in (1, -1):
            setattr(c, name, old + sign * step)
            loss.append(float((c.forward(y_in=None)[0].double() * w.double()).sum()))
        setattr(c, name, old)
        want = float((grad.double() * step.double()).sum())
        size = float((grad.double() * step.double()).abs().sum())
        # 72 x 88 products of 10 + 88 terms in fp32 on both sides: 1e-5 of the sum of magnitudes is 100 of them in a row
        assert abs((loss[0] - loss[1]) / 2 - want) <= 1e-5 * size, name


def test_the_same_bits_again_on_another_stream_and_from_a_graph():
    c = Case(1500, 264, 520, 48, 5, "bf16", ranks=True)
    ws = c.workspace()
    y, h = c.forward(ws=ws)
    dx, dq, dp = c.backward(h, ws=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y2, h2 = c.forward(ws=ws)
        again = c.backward(h2, ws=ws)
    side.synchronize()
    for a, b in zip((y, h, dx, dq, dp), (y2, h2) + again):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y3, h3 = c.forward(ws=ws)
        third = c.backward(h3, ws=ws)
    for _ in range(3):
        for t in (y3, h3) + third:
            t.fill_(float("nan"))
        c.forward()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((y, h, dx, dq, dp), (y3, h3) + third):
            assert torch.equal(a, b)


def test_no_rows_give_zero_gradients():
    c = Case(4, 16, 24, 3, 2, "f32")
    empty = lambda k: torch.empty(0, k, device=DEV)  # noqa: E731
    dq, dp = (torch.full((2, 3, k), 5.0, device=DEV) for k in (24, 16))
    ids = torch.empty(0, device=DEV, dtype=torch.int32)
    ws = torch.empty(dlcx.dlcx_adapter_workspace_bytes(c.d, 0), device=DEV, dtype=torch.uint8)
    dlcx.dlcx_adapter_forward(c.d, empty(24), ids, c.qd, c.pd, empty(16), empty(16), empty(3), ws)
    dlcx.dlcx_adapter_backward(c.d, empty(24), empty(16), ids, c.qd, c.pd, empty(3), empty(24), empty(24), dq, dp, ws)
    assert not dq.any() and not dp.any()


def test_a_view_that_passes_32_bits():
    # the rows of a large activation, 2^28 elements apart: the last one begins past 2^31 elements
    c = Case(9, 64, 64, 8, 2, "bf16", outside=False)
    far = torch.empty(9 * (1 << 28), device=DEV, dtype=torch.bfloat16)[:9 * (1 << 28)].view(9, 1 << 28)[:, :64]
    far.copy_(c.x)
    y, h = c.forward()
    c.x = far
    y2, h2 = c.forward()
    assert torch.equal(y, y2) and torch.equal(h, h2)


def test_adapters_that_were_trained_fold_into_an_error_buffer():
    # the layout of the factors is that of every factor of the library: e <- e - P Q^T
    m, n, r = 128, 256, 16
    c = Case(64, m, n, r, 1, "f32", order="one")
    e = torch.randn(m, n, device=DEV)
    want = e.double().cpu() - c.p[0].double().t() @ c.q[0].double()
    d = dlcx.desc(m, n, r, 4, 64, dlcx.MMA_F32)
    ws = torch.empty(dlcx.dlcx_workspace_bytes(d, 1), device=DEV, dtype=torch.uint8)
    dlcx.dlcx_decompress(d, c.pd[0], c.qd[0], None, [e], workspace=ws)
    assert float((e.double().cpu() - want).norm() / want.norm()) < 1e-5


def test_wrong_tensors_are_refused_before_anything_runs():
    c = Case(20, 64, 72, 8, 2, "bf16")
    y, h = c.out(c.y_in), torch.empty(c.rows, c.r, device=DEV)
    good = dict(d=c.d, x=c.x, ids=c.idd, q=c.qd, p=c.pd, y_in=c.y_in, y_out=y, h_out=h, workspace=c.workspace())
    bad = [dict(x=c.x.float()), dict(x=c.x.t()), dict(x=c.x[:, :71]), dict(ids=c.idd.long()), dict(ids=c.idd[:19]),
           dict(q=c.qd[:1]), dict(p=c.pd.float()), dict(y_out=y[:, :63]), dict(y_in=c.y_in[:19]), dict(h_out=h[:19]),
           dict(workspace=good["workspace"][:-1]), dict(x=c.x.cpu()), dict(x=c.x[:1].expand(20, -1)),
           dict(h_out=h.to(torch.bfloat16))]
    for change in bad:
        with pytest.raises(ValueError):
            dlcx.dlcx_adapter_forward(**{**good, **change})
    big = dlcx.adapter_desc(64, 72, 300, 2)
    with pytest.raises((ValueError, dlcx.DlcxError)):
        dlcx.dlcx_adapter_forward(**{**good, "d": big})
