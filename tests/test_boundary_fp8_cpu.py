"""What the calls around the projection in 8 bits refuse, on the host: nothing is launched, no address is read."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2506_21263_amd as dlcx
from eight_ref import CODES, nearest_codes, quantize

F = 0x10000  # aligned to 256, never read


def eight(**kw):
    return dlcx.Fp8(**{**dict(codes=F, scales=F, rows=20, cols=72, ld=128, ldscale=4), **kw})


BAD = [dict(codes=None), dict(scales=None), dict(codes=F + 8), dict(scales=F + 2), dict(ld=127), dict(ld=112), dict(ld=136),
       dict(ldscale=3), dict(ldscale=6), dict(ldscale=0), dict(rows=-1), dict(cols=-1), dict(rows=(1 << 24) + 1),
       dict(ld=(1 << 29) + 16), dict(ldscale=(1 << 29) + 4)]


def ref(a):
    return None if a is None else C.addressof(a)


def quantize_call(rows=20, cols=72, x=F, ldx=72, dtype=dlcx.F32, square=0, out="own", out_t="own"):
    out = eight() if out == "own" else out
    out_t = eight(rows=72, cols=20) if out_t == "own" else out_t
    return dlcx.lib().dlcx_fp8_quantize(rows, cols, x, ldx, dtype, square, ref(out), ref(out_t), None)


def test_quantize_arguments():
    for bad in (dict(rows=-1), dict(cols=(1 << 24) + 1), dict(x=None), dict(x=F + 2), dict(ldx=71), dict(ldx=(1 << 29) + 1),
                dict(dtype=2), dict(square=2), dict(out=None, out_t=None), dict(out=eight(rows=21)), dict(out=eight(cols=71)),
                dict(out_t=eight()), dict(out_t=eight(rows=72, cols=21))):
        assert quantize_call(**bad) == dlcx.EINVAL, bad
    for bad in BAD:
        assert quantize_call(out=eight(**bad)) == dlcx.EINVAL, bad
    assert quantize_call(rows=0, x=None, out=eight(rows=0, codes=None), out_t=eight(rows=72, cols=0)) == dlcx.OK


def test_decode_arguments():
    L = dlcx.lib()
    for bad in BAD:
        assert L.dlcx_fp8_decode(ref(eight(**bad)), F, 72, dlcx.F32, None) == dlcx.EINVAL, bad
    for bad in ((None, F, 72, 0), (ref(eight()), None, 72, 0), (ref(eight()), F + 2, 72, 0), (ref(eight()), F, 71, 0),
                (ref(eight()), F, 72, 2)):
        assert L.dlcx_fp8_decode(*bad, None) == dlcx.EINVAL
    assert L.dlcx_fp8_decode(ref(eight(rows=0)), None, 72, 0, None) == dlcx.OK


def test_product_arguments():
    L = dlcx.lib()

    def product(x=None, w=None, y_in=F, ldi=30, y=2 * F, ldo=30, dtype=dlcx.F32, ws=F):
        return L.dlcx_fp8_product(ref(x or eight()), ref(w or eight(rows=30)), y_in, ldi, y, ldo, dtype, ws, None)

    for bad in BAD:
        if "rows" not in bad:
            assert product(x=eight(**bad)) == dlcx.EINVAL and product(w=eight(**{**dict(rows=30), **bad})) == dlcx.EINVAL, bad
    for bad in (dict(w=eight(rows=30, cols=73)), dict(y=None), dict(y=2 * F + 2), dict(ldo=29), dict(y_in=F + 2), dict(ldi=29),
                dict(y_in=2 * F, ldi=31), dict(dtype=2), dict(ws=None), dict(ws=F + 16), dict(ldo=(1 << 29) + 1)):
        assert product(**bad) == dlcx.EINVAL, bad
    assert product(x=eight(rows=0), y=None, ws=None) == dlcx.OK
    for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, (1 << 24) + 1)):
        assert dlcx.dlcx_fp8_product_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("m,n", [(1, 1), (2048, 2048), (28672, 8192), (1021, 4133), (64, 100000), (8192, 28672)])
def test_a_workspace_serves_fewer_rows(m, n):
    rows = sorted({2 ** k + e for k in range(15) for e in (-1, 0, 1)} | {0, 17, 33, 4095, 9999})
    size = [dlcx.dlcx_fp8_product_workspace_bytes(t, m, n) for t in rows]
    assert size == sorted(size) and size[0] > 0
    norm = [dlcx.dlcx_rms_norm_workspace_bytes(t, n) for t in rows]
    assert norm == sorted(norm) and norm[0] > 0


def test_norm_arguments():
    L = dlcx.lib()

    def norm(rows=20, n=72, dtype=dlcx.F32, x=F, ldx=72, r=2 * F, ldr=72, w=F, eps=1e-5, s=3 * F, lds=72, y=4 * F, ldy=72, y8="own",
             rstd=F):
        return L.dlcx_rms_norm(rows, n, dtype, x, ldx, r, ldr, w, eps, s, lds, y, ldy, ref(eight() if y8 == "own" else y8), rstd, None)

    nan = float("nan")
    for bad in (dict(rows=-1), dict(n=0), dict(n=(1 << 24) + 1), dict(dtype=2), dict(x=None), dict(x=F + 2), dict(ldx=71),
                dict(r=None), dict(s=None), dict(r=F + 2), dict(ldr=71), dict(s=F + 1), dict(lds=71), dict(w=None), dict(w=F + 2),
                dict(eps=nan), dict(eps=-1.0), dict(y=F + 2), dict(ldy=71), dict(rstd=F + 2), dict(y=None, y8=None),
                dict(s=F, lds=73), dict(s=2 * F, lds=80), dict(y8=eight(rows=19)), dict(y8=eight(cols=71))):
        assert norm(**bad) == dlcx.EINVAL, bad
    for bad in BAD:
        assert norm(y8=eight(**bad)) == dlcx.EINVAL, bad
    assert norm(rows=0, x=None, y8=None) == dlcx.OK

    def backward(rows=20, n=72, dtype=dlcx.F32, x=F, ldx=72, w=F, rstd=F, dy=2 * F, lddy=72, di=3 * F, ldi=72, do=4 * F, ldo=72, dw=F, ws=F):
        return L.dlcx_rms_norm_backward(rows, n, dtype, x, ldx, w, rstd, dy, lddy, di, ldi, do, ldo, dw, ws, None)

    for bad in (dict(rows=-1), dict(n=0), dict(dtype=-1), dict(x=None), dict(x=F + 2), dict(ldx=71), dict(w=None), dict(w=F + 2),
                dict(rstd=None), dict(rstd=F + 2), dict(dy=None), dict(lddy=71), dict(di=3 * F + 1), dict(ldi=71), dict(do=None),
                dict(ldo=71), dict(dw=None), dict(dw=F + 2), dict(ws=None), dict(ws=F + 16), dict(do=F, ldo=73), dict(do=2 * F, ldo=73),
                dict(do=3 * F, ldo=73)):
        assert backward(**bad) == dlcx.EINVAL, bad
    assert dlcx.dlcx_rms_norm_workspace_bytes(-1, 5) == 0 and dlcx.dlcx_rms_norm_workspace_bytes(5, 0) == 0


def test_dropout_arguments():
    L = dlcx.lib()

    def drop(rows=20, cols=72, dtype=dlcx.F32, x=F, ldx=72, yi=2 * F, ldi=72, yo=3 * F, ldo=72, p=0.1, more=F):
        return L.dlcx_dropout(rows, cols, dtype, x, ldx, yi, ldi, yo, ldo, p, 1, 2, more, None)

    nan = float("nan")
    for bad in (dict(rows=-1), dict(cols=(1 << 24) + 1), dict(dtype=2), dict(x=None), dict(x=F + 2), dict(ldx=71), dict(yi=F + 1),
                dict(ldi=71), dict(yo=None), dict(ldo=71), dict(p=-0.1), dict(p=1.0), dict(p=nan), dict(p=1 - 2.0 ** -18),
                dict(more=F + 4), dict(yo=F, ldo=73), dict(yo=2 * F, ldo=73)):
        assert drop(**bad) == dlcx.EINVAL, bad
    assert drop(rows=0, x=None) == dlcx.OK


def test_pitches():
    assert [dlcx.dlcx_fp8_code_pitch(c) for c in (0, 1, 128, 129)] == [0, 128, 128, 256]
    assert [dlcx.dlcx_fp8_scale_pitch(c) for c in (0, 1, 512, 513)] == [0, 4, 4, 8]
    assert dlcx.dlcx_fp8_code_pitch(-1) == 0


def test_the_reference_of_the_codes():
    """What the GPU tests compare with, against torch's own conversion."""
    x = torch.cat([torch.tensor([0.0, -0.0]), torch.linspace(-448, 448, 20001), torch.randn(20000) * 2.0 ** torch.randint(-9, 7, (20000,))])
    x = x.clamp(-448, 448)
    assert np.array_equal(nearest_codes(x.double().numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(v, nan=1e9), np.nan_to_num(CODES, nan=1e9))
    c, s = quantize(np.array([[449.0] + [1.0] * 200, [448.0] * 201]))
    assert s.tolist() == [[128, 119], [127, 127]] and c[0, 0] == 0x76 and c[1, 0] == 0x7e
