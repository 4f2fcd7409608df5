"""Norm and gradient of as many short rows as the header allows, against the formulas in 64 bits, on the GPU.

u = 2^-24.  A sum of n <= 7 terms is off by n u of their magnitudes, a root and a quotient by u each, a product by u."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from eight_ref import DEV, HALF, TYPES, U

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.mark.parametrize("rows,n,dtype", [(1 << 22, 5, "f32"), ((1 << 23) - 1, 3, "bf16"), (1 << 24, 1, "bf16")])
def test_norm_of_many_short_rows(rows, n, dtype):
    dt = TYPES[dtype]
    gen = torch.Generator(device=DEV).manual_seed(n)
    x, r, dy = (torch.randn(rows, n, generator=gen, device=DEV).to(dt) for _ in range(3))
    w = (1 + 0.3 * torch.randn(n, generator=gen, device=DEV)).to(dt)
    want_sum = (x.double() + r.double()).to(dt)
    y, total, rstd = torch.full_like(x, 9.0), torch.full_like(x, 9.0), torch.full((rows,), 9.0, device=DEV)
    dlcx.dlcx_rms_norm(x, w, EPS, residual=r, sum_out=total, y_out=y, rstd_out=rstd)
    assert torch.equal(total, want_sum)
    s, wv = want_sum.double(), w.double()
    want = 1 / torch.sqrt((s * s).mean(1) + EPS)
    off = (n + 6) * U
    assert bool(((rstd.double() - want).abs() <= off * want).all())
    v = s * want[:, None] * wv
    assert bool(((y.double() - v).abs() <= v.abs() * (off + 3 * U + (1.01 * HALF[dt] if dtype == "bf16" else 0)) + 1e-40).all())

    dx, dw = torch.full_like(x, 9.0), torch.full((n,), 9.0, device=DEV)
    ws = torch.empty(dlcx.dlcx_rms_norm_workspace_bytes(rows, n), device=DEV, dtype=torch.uint8).fill_(255)
    dlcx.dlcx_rms_norm_backward(total, w, rstd, dy, r, dx, dw, ws)
    h, g = s * rstd.double()[:, None], dy.double() * wv
    dot, most = (g * h).mean(1, keepdim=True), (g * h).abs().mean(1, keepdim=True)
    want = r.double() + rstd.double()[:, None] * (g - h * dot)
    lim = rstd.double()[:, None] * (g.abs() * 6 * U + h.abs() * ((n + 12) * U * most)) + 2 * U * r.double().abs()
    if dtype == "bf16":
        lim = lim + 1.01 * HALF[dt] * want.abs()
    assert bool(((dx.double() - want).abs() <= lim + 1e-40).all())
    # at most 1024 parts of rows / 1024 terms one after the other, then the parts
    terms = dy.double() * h
    assert bool(((dw.double() - terms.sum(0)).abs() <= (rows / 1024 + 1100) * U * terms.abs().sum(0)).all())
