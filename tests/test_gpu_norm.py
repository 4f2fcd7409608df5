"""Root-mean-square norm and its gradient against the formulas in 64 bits, element by element.

u = 2^-24.  The sum of n squares goes through at most n / 64 + 40 additions one after the other (a lane's own, then the
tree), so it is off by (n / 64 + 40) u of itself (all terms are positive), rstd by half of that and 3 u, y by 3 u more
and its rounding.  Sums with signs: the same number of steps times the sum of magnitudes."""
import numpy as np
import pytest
import torch

import paper_2506_21263_amd as dlcx
from eight_ref import CODES, DEV, HALF, TYPES, U, around, f64, matrix, scale_exponents

pytestmark = pytest.mark.gpu
EPS = 1e-5


def steps(n):
    return n / 64 + 40


def forward(x, w, residual=None, y=True, y8=False, in_place=False):
    rows, n = x.shape
    out = dict(rstd=torch.full((rows,), 9.0, device=DEV))
    if residual is not None:
        out["sum"] = x if in_place else torch.full_like(x, 9.0)
    if y:
        out["y"] = torch.full((rows, n), 9.0, device=DEV, dtype=x.dtype)
    if y8:
        out["y8"] = dlcx.fp8_empty(rows, n, DEV)
        for t in out["y8"].held:
            t.view(torch.uint8).fill_(0x55)
    dlcx.dlcx_rms_norm(x, w, EPS, residual=residual, sum_out=out.get("sum"), y_out=out.get("y"), y8_out=out.get("y8"),
                       rstd_out=out["rstd"])
    return out


def check_forward(rows, n, dtype, residual, y, y8, pad=0, shift=0, std=1.0, in_place=False):
    gen = torch.Generator().manual_seed(rows + 3 * n)
    dt = TYPES[dtype]
    x, w = matrix(gen, rows, n, dt, std, pad, shift), (1 + 0.3 * torch.randn(n, generator=gen)).to(dt).to(DEV)
    r = matrix(gen, rows, n, dt, std, pad, shift) if residual else None
    want_sum = (f64(x) + f64(r)) if residual else f64(x)
    out = forward(x, w, r, y, y8, in_place)
    s = want_sum
    if residual:
        s = f64(torch.from_numpy(want_sum).to(dt))                 # fp32: the sum of two is rounded once
        assert np.array_equal(f64(out["sum"]), s)
    rstd = 1 / np.sqrt((s * s).mean(1) + EPS)
    off = steps(n) * U / 2 + 4 * U
    assert (np.abs(f64(out["rstd"]) - rstd) <= off * rstd).all()
    v = s * rstd[:, None] * f64(w)
    off += 3 * U
    if y:
        assert (np.abs(f64(out["y"]) - v) <= np.abs(v) * (off + (1.01 * HALF[dt] if dtype == "bf16" else 0)) + 1e-40).all()
    if y8:
        codes, scales = (t.view(torch.uint8).cpu().numpy() for t in out["y8"].held)
        assert not codes[:, n:].any()
        for b in range(-(-n // 128)):
            part, k = v[:, b * 128:(b + 1) * 128], scales[:, b].astype(np.int64) - 127
            top = np.abs(part).max(1)
            low, high = (scale_exponents(top * (1 + e)) for e in (-off, off))
            assert ((k >= low) & (k <= high)).all()
            got = np.ldexp(CODES[codes[:, b * 128:b * 128 + part.shape[1]]], k[:, None])
            half = np.maximum(np.abs(part) * (1 + off) * 2.0 ** -4, np.ldexp(1.0, k - 10)[:, None])
            assert (np.abs(got - part) <= half + off * np.abs(part)).all()
    if pad or shift:
        assert bool(around(x, rows, n).isnan().all())


SHAPES = [(1, 1), (1, 2048), (3, 7), (5, 512), (6, 513), (2, 1021), (9, 2050), (4, 4096), (5, 4100), (3, 8192), (2, 8195),
          (3, 16384), (2, 20000), (2, 32768), (3, 32769), (2, 40001), (300, 130)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual,y,y8", [(False, True, False), (True, False, True), (True, True, True)])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_norm(rows, n, dtype, residual, y, y8):
    check_forward(rows, n, dtype, residual, y, y8)


@pytest.mark.parametrize("n", [5, 600, 2050, 9001, 33001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_views(n, dtype):
    """Rows that are apart and begin anywhere; the sum over x itself; small and large values."""
    check_forward(6, n, dtype, True, True, True, pad=3, shift=1, in_place=True)
    check_forward(6, n, dtype, False, True, True, pad=2, shift=2, std=1e-3)
    check_forward(6, n, dtype, True, True, False, pad=1, shift=3, std=1e4)


def test_rows_of_zeros_and_of_nan():
    x = torch.randn(7, 700, device=DEV)
    x[2], x[4, 9] = 0.0, float("nan")
    out = forward(x, torch.ones(700, device=DEV), y8=True)
    assert not bool(out["y"][2].any()) and bool(out["y"][4].isnan().all())
    assert bool(out["y"][[0, 1, 2, 3, 5, 6]].isfinite().all())
    codes = out["y8"].held[0].view(torch.uint8)
    assert not bool(codes[2].any()) and bool(((codes[4, :700] & 127) == 127).all())
    assert abs(float(out["rstd"][2]) - EPS ** -0.5) <= 4 * U * EPS ** -0.5


# ---- the gradient -----------------------------------------------------------------------------
def check_backward(rows, n, dtype, residual, pad=0, shift=0, alias=None):
    gen = torch.Generator().manual_seed(rows + 5 * n)
    dt = TYPES[dtype]
    x, dy = matrix(gen, rows, n, dt, 2.0, pad, shift), matrix(gen, rows, n, dt, 0.1, pad, shift)
    dx_in = matrix(gen, rows, n, dt, 0.1, pad, shift) if residual else None
    w = (1 + 0.3 * torch.randn(n, generator=gen)).to(dt).to(DEV)
    rstd = torch.from_numpy(1 / np.sqrt((f64(x) ** 2).mean(1) + EPS)).float().to(DEV)
    xv, dyv, wv, rv, base = f64(x), f64(dy), f64(w), f64(rstd)[:, None], f64(dx_in) if residual else 0.0
    dx = dict(x=x, dy=dy, dx_in=dx_in).get(alias)
    if dx is None:
        dx = matrix(gen, rows, n, dt, 1.0, pad, shift)
    dw = torch.full((n,), 9.0, device=DEV)
    ws = torch.empty(dlcx.dlcx_rms_norm_workspace_bytes(rows, n), device=DEV, dtype=torch.uint8).fill_(255)
    dlcx.dlcx_rms_norm_backward(x, w, rstd, dy, dx_in, dx, dw, ws)
    h, g = xv * rv, dyv * wv
    dot = (g * h).mean(1, keepdims=True)
    want = base + rv * (g - h * dot)
    dot_off = (steps(n) + 6) * U * np.abs(g * h).mean(1, keepdims=True)
    off = rv * (np.abs(g) * 6 * U + np.abs(h) * (dot_off + 6 * U * np.abs(dot))) + 2 * U * np.abs(base)
    if dtype == "bf16":
        off = off + 1.01 * HALF[dt] * np.abs(want)
    assert (np.abs(f64(dx) - want) <= off + 1e-40).all()
    assert (np.abs(f64(dw) - (dyv * h).sum(0)) <= (rows + 30) * U * np.abs(dyv * h).sum(0) + 1e-40).all()
    if pad or shift:
        assert bool(around(dx, rows, n).isnan().all())


@pytest.mark.parametrize("dtype,residual", [("f32", False), ("bf16", True), ("f32", True), ("bf16", False)])
@pytest.mark.parametrize("rows,n", SHAPES + [(2100, 300), (1500, 2050), (300, 33000)])
def test_gradient(rows, n, dtype, residual):
    check_backward(rows, n, dtype, residual)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(9001, 5), (5003, 8), (9001, 130), (4099, 512), (2500, 1023)])
def test_gradient_of_many_short_rows(rows, n, dtype):
    check_backward(rows, n, dtype, True, pad=1, shift=1)


@pytest.mark.parametrize("alias", ["x", "dy", "dx_in"])
@pytest.mark.parametrize("n", [5, 600, 2050, 9001, 33001])
def test_gradient_of_views_in_place(n, alias):
    check_backward(6, n, "bf16", True, pad=3, shift=1, alias=alias)
    check_backward(5, n, "f32", True, pad=1, shift=3, alias=alias)


def test_no_rows():
    """An empty batch: tensors without elements have no address."""
    x, w = torch.empty(0, 300, device=DEV), torch.ones(300, device=DEV)
    out = forward(x, w, torch.empty(0, 300, device=DEV), y8=True)
    assert out["y"].shape == (0, 300)
    y = torch.empty(0, 7, device=DEV)
    w8 = dlcx.fp8_empty(7, 300, DEV)
    ws = torch.empty(dlcx.dlcx_fp8_product_workspace_bytes(0, 7, 300), device=DEV, dtype=torch.uint8)
    dlcx.dlcx_fp8_quantize(x, out["y8"], dlcx.fp8_empty(300, 0, DEV))
    dlcx.dlcx_fp8_product(out["y8"], w8, None, y, ws)
    dlcx.dlcx_dropout(x, None, x, 0.5, 1)


def test_gradient_without_rows():
    dw = torch.full((300,), 9.0, device=DEV)
    x = torch.empty(0, 300, device=DEV)
    ws = torch.empty(dlcx.dlcx_rms_norm_workspace_bytes(0, 300), device=DEV, dtype=torch.uint8)
    dlcx.dlcx_rms_norm_backward(x, torch.ones(300, device=DEV), torch.empty(0, device=DEV), x, None, x, dw, ws)
    assert not bool(dw.any())


def test_gradient_against_differences():
    """Central differences of sum(c y) along a direction, both sides from the kernel.  They may differ from the gradient
    by what the same differences in 64 bits are off (the third derivative), and by y's own error on both sides."""
    gen = torch.Generator().manual_seed(11)
    rows, n, h = 5, 777, 2.0 ** -5
    x, c, w = matrix(gen, rows, n, torch.float32), matrix(gen, rows, n, torch.float32), 1 + 0.3 * torch.randn(n, generator=gen).to(DEV)
    d, dwt = matrix(gen, rows, n, torch.float32), torch.randn(n, generator=gen).to(DEV)
    out = forward(x, w)
    dx, dw = torch.empty_like(x), torch.empty(n, device=DEV)
    ws = torch.empty(dlcx.dlcx_rms_norm_workspace_bytes(rows, n), device=DEV, dtype=torch.uint8)
    dlcx.dlcx_rms_norm_backward(x, w, out["rstd"], c, None, dx, dw, ws)

    def exact(xv, wv):
        return xv / np.sqrt((xv * xv).mean(1, keepdims=True) + EPS) * wv

    for a, b, slope in ((d, torch.zeros_like(w), (f64(dx) * f64(d)).sum()), (torch.zeros_like(x), dwt, (f64(dw) * f64(dwt)).sum())):
        sides = [((x + s * h * a).contiguous(), w + s * h * b) for s in (1, -1)]
        mine = sum(s * (f64(c) * f64(forward(xx, ww)["y"])).sum() for s, (xx, ww) in zip((1, -1), sides)) / (2 * h)
        true = sum(s * (f64(c) * exact(f64(xx), f64(ww))).sum() for s, (xx, ww) in zip((1, -1), sides)) / (2 * h)
        noise = (steps(n) + 8) * U * np.abs(f64(c) * exact(f64(x), f64(w))).sum() * 2 / h
        xv, wv = f64(x), f64(w)
        r = 1 / np.sqrt((xv * xv).mean(1, keepdims=True) + EPS)
        g = f64(c) * wv
        analytic = ((r * (g - xv * r * (g * xv * r).mean(1, keepdims=True))) * f64(a)).sum() + (f64(c) * xv * r * f64(b)).sum()
        assert abs(mine - slope) <= abs(true - analytic) + noise


def test_same_bits_again_and_from_a_graph():
    gen = torch.Generator().manual_seed(12)
    rows, n = 3000, 1030
    x, dy, w = matrix(gen, rows, n, torch.bfloat16), matrix(gen, rows, n, torch.bfloat16), torch.ones(n, device=DEV).bfloat16()
    rstd, y, dx, dw = torch.empty(rows, device=DEV), torch.empty_like(x), torch.empty(rows, n, device=DEV).bfloat16(), torch.empty(n, device=DEV)
    ws = torch.empty(dlcx.dlcx_rms_norm_workspace_bytes(rows, n), device=DEV, dtype=torch.uint8)

    def both():
        dlcx.dlcx_rms_norm(x, w, EPS, y_out=y, rstd_out=rstd)
        dlcx.dlcx_rms_norm_backward(x, w, rstd, dy, None, dx, dw, ws)

    y = y.contiguous()
    both()
    want = [t.clone() for t in (y, rstd, dx, dw)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for _ in range(3):
        for t in (y, rstd, dx, dw):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, rstd, dx, dw), want))
