"""The norm, the shared projection in 8 bits, dropout and the adapters as they are used together: one step against the
same formulas in 64 bits on the values that the codes stand for, and its gradients."""
import numpy as np
import pytest
import torch

import paper_2506_21263_amd as dlcx
from eight_ref import DEV, HALF, TYPES, decode, f64, kept, matrix, quantize
from paper_2506_21263_amd import inner

pytestmark = pytest.mark.gpu


def eight(x, square=False):
    codes, scales = quantize(x, square)
    return decode(codes, scales, x.shape[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,m,n,K,r,p", [(24, 96, 200, 2, 5, 0.0), (150, 130, 257, 3, 8, 0.25), (1, 64, 512, 1, 4, 0.5)])
def test_one_step(rows, m, n, K, r, p, dtype):
    """Every stage is held to its own rounding on the inputs that the stage before gave on the GPU, so no error adds up:
    the products' terms are those of the codes, sums are off by (terms + 8) 2^-23 of their magnitudes (2^-10 where a bf16
    result takes 8-bit products), the adapter's by the same through both of its factors, and a result by half a step."""
    dt = TYPES[dtype]
    gen = torch.Generator().manual_seed(rows + m)
    x, res, dy = matrix(gen, rows, n, dt), matrix(gen, rows, n, dt), matrix(gen, rows, m, dt, 0.01)
    theta = matrix(gen, m, n, torch.float32, 0.05)
    q0 = torch.randn(K, r, n, generator=gen).to(DEV) * 0.1
    proj = inner.AdapterProjection(theta, q0, 1.5, rows, dt, base_bits=8, dropout=p, seed=77)
    p0 = torch.randn(K, r, m, generator=gen).to(DEV) * 0.1
    proj.p.copy_(p0)
    if dt == torch.bfloat16:
        proj.p_copy.copy_(p0)
    norm = inner.Norm(n, dt)
    ids = (torch.arange(rows) * K // rows).to(torch.int32).to(DEV)
    route = inner.Route(ids, K)
    xn, xn8, saved = norm.forward(x, res, eight=True)
    y, h = proj.forward(xn, route, xn8, draw=5)
    dx = proj.backward(xn, h, dy, route, draw=5)
    din = norm.backward(saved, dx, dy @ theta.to(dt) if n == m else None)

    w = eight(f64(theta), True)
    assert np.array_equal(decode(*(t.view(torch.uint8).cpu().numpy() for t in proj.base8.held), n), w)
    assert np.array_equal(decode(*(t.view(torch.uint8).cpu().numpy() for t in proj.base8_t.held), m), w.T)
    mask = kept(rows * n, p, 77, 5).reshape(rows, n) if p else np.ones((rows, n))
    keep = 1 - round(p * 65536) / 65536
    half = HALF[dt] * 1.01
    xd = f64(torch.from_numpy(f64(xn) * mask / keep).to(dt))
    x8 = decode(*(t.view(torch.uint8).cpu().numpy() for t in xn8.held), n)
    at = ids.cpu().numpy()
    Q, P = (f64(t) for t in (proj.q_copy, proj.p_copy))
    slack = (n + m + 3 * r + 16) * 2.0 ** -23
    cut = 2.0 ** -10 if dtype == "bf16" else 0.0
    # forward: the product rounded to dt, the adapter added to that and rounded again; xd is rounded too
    hx = np.einsum("ti,tci->tc", xd, Q[at])
    base = x8 @ w.T
    want = base + 1.5 * np.einsum("tc,tcj->tj", hx, P[at])
    mag = np.abs(x8) @ np.abs(w).T + 1.5 * np.einsum("tc,tcj->tj", np.einsum("ti,tci->tc", np.abs(xd), np.abs(Q[at])), np.abs(P[at]))
    lost = cut * (np.abs(x8) @ np.abs(w).T) + (2 * half if p else 0) * mag
    assert (np.abs(f64(y) - want) <= slack * mag + lost + half * (np.abs(base) + np.abs(want))).all()
    # backward
    d = f64(dy)
    d8 = eight(d)
    g = 1.5 * np.einsum("tj,tcj->tc", d, P[at])
    base = d8 @ w
    want = base + np.einsum("tc,tci->ti", g, Q[at]) * mask / keep
    through = np.einsum("tc,tci->ti", 1.5 * np.einsum("tj,tcj->tc", np.abs(d), np.abs(P[at])), np.abs(Q[at])) * mask / keep
    mag = np.abs(d8) @ np.abs(w) + through
    lost = cut * (np.abs(d8) @ np.abs(w)) + (2 * half if p else 0) * through
    assert (np.abs(f64(dx) - want) <= slack * mag + lost + half * (np.abs(base) + np.abs(want))).all()
    # factors' gradients: g and h are off by slack of their own magnitudes, and so is the sum over the rows
    gm = 1.5 * np.einsum("tj,tcj->tc", np.abs(d), np.abs(P[at]))
    hm = 1.5 * np.einsum("ti,tci->tc", np.abs(xd), np.abs(Q[at]))
    slack += rows * 2.0 ** -23
    for a in range(K):
        mine = at == a
        for got, left, size, right in ((proj.dq[a], g, gm, xd), (proj.dp[a], 1.5 * hx, hm, d)):
            lim = (2 * slack + (2 * half if p else 0)) * (size[mine].T @ np.abs(right[mine])) + 1e-30
            assert (np.abs(f64(got) - left[mine].T @ right[mine]) <= lim).all()
    # the norm's gradient, of the dx that was there
    s, wn, r_ = f64(saved[0]), f64(norm.weight), f64(saved[1])[:, None]
    hh, gg = s * r_, f64(dx) * wn
    want = r_ * (gg - hh * (gg * hh).mean(1, keepdims=True))
    lim = (n / 64 + 60) * 2.0 ** -24 * r_ * (np.abs(gg) + np.abs(hh) * np.abs(gg * hh).mean(1, keepdims=True)) + half * np.abs(want)
    assert (np.abs(f64(din) - want) <= lim).all()


@pytest.mark.parametrize("dropout,norm,dtype", [(0.0, False, torch.bfloat16), (0.1, True, torch.bfloat16), (0.1, True, torch.float32)], ids=str)
def test_training_runs(dropout, norm, dtype):
    losses = inner.train(m=256, n=384, rows=64, inner=4, outer=3, base_bits=8, dropout=dropout, norm=norm, dtype=dtype)
    assert len(losses) == 3 and all(np.isfinite(losses))


def test_what_ran_before_is_as_it_was():
    """Without the new options the same bits as the calls themselves."""
    gen = torch.Generator().manual_seed(1)
    theta, x = matrix(gen, 64, 96, torch.float32, 0.1), matrix(gen, 20, 96, torch.bfloat16)
    proj = inner.AdapterProjection(theta, torch.randn(2, 4, 96, generator=gen).to(DEV), 1.0, 20)
    route = inner.Route((torch.arange(20) // 10).to(torch.int32).to(DEV), 2)
    y, h = proj.forward(x, route)
    assert torch.equal(y, x @ theta.to(torch.bfloat16).t())     # P is zero
    assert proj.base8 is None and proj.dropout == 0.0
