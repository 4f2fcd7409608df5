"""How many outputs a product in 8 bits may have, as the header says it: refused on the host, nothing is launched."""
import ctypes as C
import os

import pytest

import paper_2506_21263_amd as dlcx

F = 0x10000  # aligned to 256, never read


@pytest.mark.parametrize("dtype", [dlcx.F32, dlcx.BF16])
@pytest.mark.parametrize("rows,m", [(1 << 18, 1 << 18), (1 << 24, 1 << 24), (1 << 24, 1 << 12), (1 << 12, 1 << 24),
                                    ((1 << 24) - 127, (1 << 12) - 127)])
def test_products_of_too_many_outputs(rows, m, dtype):
    x, w = (dlcx.Fp8(codes=F, scales=F, rows=k, cols=72, ld=128, ldscale=4) for k in (rows, m))
    assert dlcx.lib().dlcx_fp8_product(C.addressof(x), C.addressof(w), None, m, F, m, dtype, F, None) == dlcx.EUNSUPPORTED


def test_the_header_names_the_limit():
    text = open(os.path.join(os.path.dirname(dlcx.HERE), "include", "dlcx.h")).read()
    about = text[text.index("/* y_out = y_in + x w^T: x is rows x n"):text.index("int dlcx_fp8_product(")]
    assert "DLCX_EUNSUPPORTED" in about and "2^36 outputs" in about
