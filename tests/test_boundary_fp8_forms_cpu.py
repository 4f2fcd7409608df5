"""The plan of a product in 8 bits, on the host: what it refuses, and that the forms' tests reach every kernel."""
import ctypes as C

import paper_2506_21263_amd as dlcx
from eight_forms import BF16, F32, FEW, FORMS, RING, TILES, WIDE

CODE = {F32: dlcx.F32, BF16: dlcx.BF16}


def test_sizes_take_the_form_that_they_are_meant_to():
    wrong = [(size, dtype, plan, got) for size, dtype, plan in FORMS
             for got in [dlcx.dlcx_fp8_product_plan(*size, CODE[dtype])] if got != plan]
    assert not wrong


def test_every_kernel_is_reached():
    """Result type, form, tile, and whether the sum is split (few rows and tiles of 256 x 256 never are)."""
    have = {(dtype, form, tile, splits > 1) for _, dtype, (form, tile, splits) in FORMS}
    want = {(d, FEW, kw, False) for d in CODE for kw in (1, 2, 4)}
    want |= {(d, RING, t, s) for d in CODE for t in (32, 64, 96, 128) for s in (False, True)}
    want |= {(d, TILES, t, s) for d in CODE for t in (64, 128) for s in (False, True)} | {(BF16, WIDE, 256, False)}
    assert have == want
    blocks = {-(-n // 128) % 4 for (_, _, n), _, plan in FORMS if plan[0] == WIDE}
    assert blocks == {0, 1, 2, 3}


def test_a_workspace_holds_the_splits():
    for (rows, m, n), _, (_, _, splits) in FORMS:
        if splits > 1:
            assert dlcx.dlcx_fp8_product_workspace_bytes(rows, m, n) >= splits * rows * -(-m // 4) * 16


def test_plan_arguments():
    L = dlcx.lib()
    k = C.addressof(C.c_int32())
    for bad in ((-1, 1, 1, 0, k, k, k), (1, (1 << 24) + 1, 1, 0, k, k, k), (1, 1, -1, 0, k, k, k), (1, 1, 1, 2, k, k, k),
                (1, 1, 1, 0, None, k, k), (1, 1, 1, 0, k, None, k), (1, 1, 1, 0, k, k, None)):
        assert L.dlcx_fp8_product_plan(*bad) == dlcx.EINVAL, bad
