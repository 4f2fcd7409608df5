"""Matrices in 8 bits: quantiser, what codes stand for, and the product, against the definitions.

Codes and scales have to be the same to the last bit: x times a power of two is exact, and is rounded once.  The
product's sum of n terms in fp32 is off by at most a step (2^-23) of the sum of magnitudes for each addition, whether the
matrix cores round or cut.  A bf16 result takes the cores' 8-bit products, which cut each of eight at 2^-13 of the largest
of them before they are added: seven such cuts are at most 7 2^-13 < 2^-10 of the eight's sum of magnitudes; and its
rounding is off by 2^-8 of the result."""
import numpy as np
import pytest
import torch

import paper_2506_21263_amd as dlcx
from eight_ref import CODES, DEV, HALF, TYPES, U, around, decode, f64, matrix, quantize

pytestmark = pytest.mark.gpu


def fresh(rows, cols, fill=0x55):
    a = dlcx.fp8_empty(rows, cols, DEV)
    for t in a.held:
        t.view(torch.uint8).fill_(fill)
    return a


def bytes_of(a):
    return [t.view(torch.uint8).cpu().numpy() for t in a.held]


def same(a, x, square=False):
    """The matrix in 8 bits holds what the definition gives for x, and zeros behind each row."""
    rows, cols = x.shape
    codes, scales = bytes_of(a)
    want, ws = quantize(x, square)
    assert np.array_equal(scales[:, :ws.shape[1]], ws)
    assert np.array_equal(codes[:, :cols], want)
    assert not codes[:, cols:].any()


SHAPES = [(1, 1), (1, 2048), (7, 129), (128, 128), (129, 127), (200, 640), (515, 2050), (1021, 33), (3, 5000)]


@pytest.mark.parametrize("form", ["rows", "cols", "both", "square", "square_rows", "square_cols"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize(rows, cols, dtype, form):
    gen = torch.Generator().manual_seed(rows + 3 * cols)
    x = matrix(gen, rows, cols, TYPES[dtype], pad=rows % 3, shift=cols % 4)
    x *= torch.exp(3 * torch.randn(rows, 1, generator=gen)).to(x)
    out = fresh(rows, cols) if form not in ("cols", "square_cols") else None
    out_t = fresh(cols, rows) if form not in ("rows", "square_rows") else None
    dlcx.dlcx_fp8_quantize(x, out, out_t, square="square" in form)
    if out is not None:
        same(out, f64(x), "square" in form)
    if out_t is not None:
        same(out_t, f64(x).T, "square" in form)
    for a, cols_ in ((out, cols), (out_t, rows)):
        if a is not None:
            for dt in TYPES.values():
                v = torch.full((a.rows, cols_ + 3), 7.0, device=DEV, dtype=dt)
                dlcx.dlcx_fp8_decode(a, v[:, :cols_])
                c, s = bytes_of(a)
                assert np.array_equal(f64(v[:, :cols_]), decode(c, s, cols_)) and bool((v[:, cols_:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", ["both", "square"])
@pytest.mark.parametrize("rows,cols", [(200, 3), (130, 7), (300, 8), (133, 9), (257, 135)])
def test_quantize_narrow(rows, cols, form, dtype):
    test_quantize(rows, cols, dtype, form)


def test_every_code_and_what_is_between_them():
    """Codes come back as they are, and values between two of them go to the nearest, ties to the even one."""
    v = np.sort(CODES[np.isfinite(CODES) & (CODES >= 0)])
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid.astype(np.float32), np.float32(np.inf)).astype(np.float64),
                        np.nextafter(mid.astype(np.float32), np.float32(0)).astype(np.float64)])
    x = np.concatenate([x, -x])
    x = np.concatenate([x, np.zeros(-x.size % 127)]).reshape(-1, 127)
    x = np.concatenate([np.full((x.shape[0], 1), 448.0), x], 1)   # every block has scale 1
    a = fresh(*x.shape)
    dlcx.dlcx_fp8_quantize(torch.from_numpy(x).float().to(DEV), a)
    same(a, x)


def test_scales_at_their_borders():
    """Largest values next to 448 2^k, the smallest and largest numbers, blocks of zeros."""
    f = np.float32
    tops = [f(0), f(1.75), np.nextafter(f(1.75), f(2)), np.nextafter(f(1.75), f(1)), f(448), f(2.0) ** -126, f(2.0) ** -149,
            f(2.0) ** -119, f(1.75) * f(2.0) ** -119, np.nextafter(f(1.75) * f(2.0) ** -119, f(1)), np.finfo(f).max,
            f(1.75) * f(2.0) ** 127, f(2.0) ** -118, f(3e-39)]
    x = np.zeros((len(tops), 128), f)
    rng = np.random.default_rng(0)
    for i, t in enumerate(tops):
        x[i] = (rng.uniform(-1, 1, 128) * t).astype(f)
        x[i, i] = -t
    a = fresh(*x.shape)
    dlcx.dlcx_fp8_quantize(torch.from_numpy(x).to(DEV), a)
    same(a, x.astype(np.float64))


@pytest.mark.parametrize("square", [False, True])
def test_values_that_are_not_finite(square):
    """They become NaN, and the scale is that of the others."""
    gen = torch.Generator().manual_seed(5)
    x = matrix(gen, 150, 300, torch.float32)
    x[3, 7], x[3, 8], x[4, 200], x[140, 0:128] = float("inf"), float("-inf"), float("nan"), float("nan")
    a, t = fresh(150, 300), fresh(300, 150)
    dlcx.dlcx_fp8_quantize(x, a, t, square=square)
    for m, want in ((a, f64(x)), (t, f64(x).T)):
        codes, scales = bytes_of(m)
        c, s = quantize(want, square)
        assert np.array_equal(scales[:, :s.shape[1]], s)
        bad = ~np.isfinite(want)
        assert np.array_equal(codes[:, :want.shape[1]][~bad], c[~bad])
        assert ((codes[:, :want.shape[1]][bad] & 127) == 127).all()


# ---- the product ------------------------------------------------------------------------------
def operand(gen, rows, cols, seed_scale=True):
    """Random codes and scales in all of the format (no NaN), and what they stand for."""
    a = dlcx.fp8_empty(max(rows, 0), cols, DEV)
    codes, scales = a.held
    c = torch.randint(0, 256, (rows, cols), generator=gen, dtype=torch.uint8)
    c[(c & 127) == 127] = 0x38
    codes.view(torch.uint8).zero_()
    codes.view(torch.uint8)[:, :cols] = c.to(DEV)
    s = torch.randint(118, 128, scales.shape, generator=gen, dtype=torch.uint8)
    s[:, -(-cols // 128):] = 255                                   # the pad of the scales is not read as one
    scales.copy_(s)
    return a, decode(c.numpy(), s.numpy(), cols)


def check_product(rows, m, n, dtype, add, pad=0, shift=0, alias=False):
    gen = torch.Generator().manual_seed(rows + 5 * m + 7 * n)
    x, xv = operand(gen, rows, n)
    w, wv = operand(gen, m, n)
    dt = TYPES[dtype]
    y_in = matrix(gen, rows, m, dt, 100.0, pad, shift) if add else None
    y = y_in if alias else matrix(gen, rows, m, dt, 1.0, pad, shift)
    base = f64(y_in) if add else 0.0
    ws = torch.empty(dlcx.dlcx_fp8_product_workspace_bytes(rows, m, n), device=DEV, dtype=torch.uint8).fill_(255)
    dlcx.dlcx_fp8_product(x, w, y_in, y, ws)
    got, want = f64(y), xv @ wv.T + base
    most = np.abs(xv) @ np.abs(wv).T + np.abs(base)
    bound = (n + 8) * 2.0 ** -23 * most + 1e-30
    if dtype == "bf16":
        bound += 2.0 ** -10 * most + HALF[dt] * np.abs(want) * 1.01
    assert (np.abs(got - want) <= bound).all(), np.max(np.abs(got - want) / bound)
    if pad or shift:
        assert bool(around(y, rows, m).isnan().all())
    return y


PRODUCTS = [(1, 1, 1), (1, 2048, 2048), (1, 17, 4133), (2, 130, 257), (16, 64, 128), (17, 300, 1000), (33, 1021, 515),
            (64, 96, 12000), (96, 520, 640), (128, 128, 128), (129, 257, 385), (200, 1000, 513), (256, 256, 1024),
            (300, 77, 2050), (515, 515, 1111), (1000, 130, 129), (2050, 1021, 200)]


@pytest.mark.parametrize("dtype,add", [("f32", False), ("bf16", False), ("f32", True), ("bf16", True)])
@pytest.mark.parametrize("rows,m,n", PRODUCTS)
def test_product(rows, m, n, dtype, add):
    check_product(rows, m, n, dtype, add)


@pytest.mark.parametrize("rows,m,n", [(1, 33, 300), (5, 515, 2100), (40, 131, 700), (130, 259, 129), (700, 301, 300)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_product_of_views(rows, m, n, dtype):
    """Outputs whose rows are apart and begin anywhere, in place."""
    check_product(rows, m, n, dtype, True, pad=3, shift=1, alias=True)
    check_product(rows, m, n, dtype, False, pad=5, shift=2)


@pytest.mark.parametrize("rows,m,n", [(2817, 3001, 129), (3000, 2816, 1700), (256, 32769, 515), (33000, 257, 640), (4096, 2048, 100)])
def test_large_product(rows, m, n):
    """Tiles at the edges are moved inside: every output once, in place too, and nothing around them."""
    check_product(rows, m, n, "bf16", False)
    check_product(rows, m, n, "bf16", True, pad=3, shift=1, alias=True)
    check_product(rows, m, n, "bf16", False, pad=8, shift=8)
    check_product(rows, m, n, "f32", True)


def test_product_without_terms():
    """A sum of no terms is zero: y_in comes back."""
    for rows, m, dt in ((5, 7, torch.float32), (50, 70, torch.bfloat16), (3000, 3000, torch.bfloat16)):
        x, w = dlcx.fp8_empty(rows, 0, DEV), dlcx.fp8_empty(m, 0, DEV)
        ws = torch.empty(dlcx.dlcx_fp8_product_workspace_bytes(rows, m, 0), device=DEV, dtype=torch.uint8)
        y_in, y = torch.randn(rows, m, device=DEV).to(dt), torch.full((rows, m), 9.0, device=DEV, dtype=dt)
        dlcx.dlcx_fp8_product(x, w, y_in, y, ws)
        assert torch.equal(y, y_in)
        dlcx.dlcx_fp8_product(x, w, None, y, ws)
        assert not bool(y.any())


@pytest.mark.parametrize("rows", [1, 20, 300])
def test_extreme_scales(rows):
    """Scales next to both ends of a byte's range: 2^-127 beside 2^100, and a result that no fp32 holds."""
    gen = torch.Generator().manual_seed(1)
    x, _ = operand(gen, rows, 256)
    w, _ = operand(gen, 40, 256)
    x.held[1].fill_(0)
    w.held[1].fill_(227)
    y = torch.empty(rows, 40, device=DEV)
    ws = torch.empty(dlcx.dlcx_fp8_product_workspace_bytes(rows, 40, 256), device=DEV, dtype=torch.uint8)
    dlcx.dlcx_fp8_product(x, w, None, y, ws)
    xv, wv = (decode(*bytes_of(a), 256) for a in (x, w))
    assert (np.abs(f64(y) - xv @ wv.T) <= 264 * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T)).all()
    x.held[1].fill_(254)
    for t in (x, w):
        t.held[0].view(torch.uint8).fill_(0x7e)                    # 448 2^127 448 2^100
    dlcx.dlcx_fp8_product(x, w, None, y, ws)
    assert bool((y == float("inf")).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,m,n", [(1, 90, 1100), (20, 90, 1100), (300, 130, 1100), (700, 700, 1100), (4096, 2048, 300)])
def test_scales_far_apart(rows, m, n, dtype):
    """Scales from 2^-117 to 2^73, another for every block of a row: the smallest products vanish beside the largest.  What
    fp32 cannot hold (below 2^-126 each) is in the bound's last term."""
    gen = torch.Generator().manual_seed(4)
    x, _ = operand(gen, rows, n)
    w, _ = operand(gen, m, n)
    for a, low, high in ((x, 10, 121), (w, 40, 201)):
        s = a.held[1]
        s.copy_(torch.randint(low, high, s.shape, generator=gen, dtype=torch.uint8))
        s[::3] = 127                                               # some rows' are all near 1
    xv, wv = (decode(*bytes_of(a), n) for a in (x, w))
    y = torch.empty(rows, m, device=DEV, dtype=TYPES[dtype])
    ws = torch.empty(dlcx.dlcx_fp8_product_workspace_bytes(rows, m, n), device=DEV, dtype=torch.uint8)
    dlcx.dlcx_fp8_product(x, w, None, y, ws)
    want, most = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    bound = (n + 8) * 2.0 ** -23 * most + n * 2.0 ** -126
    if dtype == "bf16":
        bound += 2.0 ** -10 * most + HALF[y.dtype] * np.abs(want) * 1.01
    assert (np.abs(f64(y) - want) <= bound).all()


@pytest.mark.parametrize("rows", [1, 20, 300])
def test_a_nan_stays_in_its_row_and_column(rows):
    gen = torch.Generator().manual_seed(2)
    x, xv = operand(gen, rows, 400)
    w, wv = operand(gen, 50, 400)
    x.held[0].view(torch.uint8)[rows - 1, 399] = 0x7f
    w.held[0].view(torch.uint8)[7, 0] = 0xff
    y = torch.empty(rows, 50, device=DEV)
    ws = torch.empty(dlcx.dlcx_fp8_product_workspace_bytes(rows, 50, 400), device=DEV, dtype=torch.uint8)
    dlcx.dlcx_fp8_product(x, w, None, y, ws)
    bad = torch.zeros(rows, 50, dtype=torch.bool)
    bad[rows - 1], bad[:, 7] = True, True
    assert torch.equal(y.isnan().cpu(), bad)
    ok = ~bad.numpy()
    assert (np.abs(f64(y) - xv @ wv.T) <= 408 * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T))[ok].all()


def test_a_projection_and_its_gradients():
    """y, dx and dw of a projection from the three products, against those of the same codes in 64 bits, and the
    gradients against differences of y: y is linear in x and w, so a difference is exact but for its rounding."""
    gen = torch.Generator().manual_seed(3)
    rows, m, n = 150, 200, 330
    x, w, dy = (matrix(gen, *s, torch.float32) for s in ((rows, n), (m, n), (rows, m)))
    x8, xt, w8, wt, dy8, dyt = (fresh(*s) for s in ((rows, n), (n, rows), (m, n), (n, m), (rows, m), (m, rows)))
    dlcx.dlcx_fp8_quantize(x, x8, xt)
    dlcx.dlcx_fp8_quantize(w, w8, wt, square=True)
    dlcx.dlcx_fp8_quantize(dy, dy8, dyt)
    ws = torch.empty(1 << 25, device=DEV, dtype=torch.uint8)
    y, dx, dw = (torch.empty(*s, device=DEV) for s in ((rows, m), (rows, n), (m, n)))
    dlcx.dlcx_fp8_product(x8, w8, None, y, ws)
    dlcx.dlcx_fp8_product(dy8, wt, None, dx, ws)
    dlcx.dlcx_fp8_product(dyt, xt, None, dw, ws)
    v = {k: decode(*bytes_of(a), a.cols) for k, a in dict(x=x8, xt=xt, w=w8, wt=wt, dy=dy8, dyt=dyt).items()}
    assert np.array_equal(v["w"], v["wt"].T)
    for got, a, b in ((y, v["x"], v["w"]), (dx, v["dy"], v["wt"]), (dw, v["dyt"], v["xt"])):
        assert (np.abs(f64(got) - a @ b.T) <= (a.shape[1] + 8) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)).all()
    # sum of dy (y(x + d) - y(x)) for a step d that is exact in the codes: one element of x to the next code up
    codes = x8.held[0].view(torch.uint8)
    i, j = 11, 57
    before = f64(y)
    codes[i, j] = 0x30 if int(codes[i, j]) != 0x30 else 0x31
    dlcx.dlcx_fp8_product(x8, w8, None, y, ws)
    step = decode(*bytes_of(x8), n)[i, j] - v["x"][i, j]
    rise = ((f64(y) - before)[i] * v["dy"][i]).sum()
    slack = 2 * (n + 8) * 2.0 ** -23 * ((np.abs(v["x"][i]) + abs(step)) @ np.abs(v["w"]).T @ np.abs(v["dy"][i]))
    slack += abs(step) * (m + 8) * 2.0 ** -23 * (np.abs(v["dy"][i]) @ np.abs(v["w"][:, j]))
    assert abs(rise - step * float(dx[i, j])) <= slack


def test_rows_far_apart():
    """Codes whose rows are 2^28 bytes apart, the last ones past 2^32."""
    gen = torch.Generator().manual_seed(4)
    rows, n, ld = 18, 200, 1 << 28
    codes = torch.empty((rows - 1) * ld + 256, device=DEV, dtype=torch.uint8)
    view = torch.as_strided(codes, (rows, 256), (ld, 1))
    x, xv = operand(gen, rows, n)
    view.copy_(x.held[0].view(torch.uint8))
    far = dlcx.fp8(view, x.held[1], n)
    w, wv = operand(gen, 33, n)
    y = torch.empty(rows, 33, device=DEV)
    ws = torch.empty(1 << 24, device=DEV, dtype=torch.uint8)
    dlcx.dlcx_fp8_product(far, w, None, y, ws)
    assert (np.abs(f64(y) - xv @ wv.T) <= (n + 8) * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T)).all()
    dlcx.dlcx_fp8_product(w, far, None, torch.empty(33, rows, device=DEV), ws)
    out = torch.empty(rows, n, device=DEV)
    dlcx.dlcx_fp8_decode(far, out)
    assert np.array_equal(f64(out), xv)
    view.fill_(0)
    dlcx.dlcx_fp8_quantize(out, far)
    same_codes, _ = quantize(xv)
    assert np.array_equal(view.cpu().numpy()[:, :n], same_codes)


def test_same_bits_again_on_another_stream_and_from_a_graph():
    gen = torch.Generator().manual_seed(6)
    cases = []
    for rows, m, n in ((3, 500, 2100), (60, 300, 4000), (700, 640, 900)):
        (x, _), (w, _) = operand(gen, rows, n), operand(gen, m, n)
        ws = torch.empty(dlcx.dlcx_fp8_product_workspace_bytes(rows, m, n), device=DEV, dtype=torch.uint8)
        cases.append((x, w, torch.empty(rows, m, device=DEV), ws))
    want = []
    for x, w, y, ws in cases:
        dlcx.dlcx_fp8_product(x, w, None, y, ws)
        want.append(y.clone())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for (x, w, y, ws), v in zip(cases, want):
        y.zero_()
        s.wait_stream(torch.cuda.current_stream())
        dlcx.dlcx_fp8_product(x, w, None, y, ws, stream=s)
        s.synchronize()
        assert torch.equal(y, v)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for x, w, y, ws in cases:
            dlcx.dlcx_fp8_product(x, w, None, y, ws)
    for _ in range(3):
        for _, _, y, ws in cases:
            y.zero_()
            ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, v) for (_, _, y, _), v in zip(cases, want))
