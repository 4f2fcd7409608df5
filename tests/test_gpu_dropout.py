"""Dropout against its definition: the mask to the last bit, values within their rounding (u = 2^-24 for the product and
the sum each, 2^-8 where the result is bf16)."""
import numpy as np
import pytest
import torch

import paper_2506_21263_amd as dlcx
from eight_ref import DEV, HALF, TYPES, U, around, f64, kept, matrix

pytestmark = pytest.mark.gpu
SEED, OFFSET = 0x9E3779B97F4A7C15, (5 << 40) + 12345


def check(rows, cols, dtype, p, add, pad=0, shift=0, alias=None, seed=SEED, offset=OFFSET, more=None):
    gen = torch.Generator().manual_seed(rows + 3 * cols)
    dt = TYPES[dtype]
    x = matrix(gen, rows, cols, dt, 1.0, pad, shift)
    y_in = matrix(gen, rows, cols, dt, 1.0, pad, shift) if add else None
    xv, base = f64(x), f64(y_in) if add else np.zeros((rows, cols))
    y = x if alias == "x" else y_in if alias == "y_in" else matrix(gen, rows, cols, dt, 1.0, pad, shift)
    extra = None if more is None else torch.tensor([more], device=DEV, dtype=torch.int64)
    dlcx.dlcx_dropout(x, y_in, y, p, seed, offset, extra)
    mask = kept(rows * cols, p, seed, (offset + (more or 0)) % 2 ** 64).reshape(rows, cols)
    scaled = xv * mask / (1 - round(p * 65536) / 65536)
    want = base + scaled
    off = 3 * U * (np.abs(base) + np.abs(scaled)) + (1.01 * HALF[dt] * np.abs(want) if dtype == "bf16" else 0)
    got = f64(y)
    assert (np.abs(got - want) <= off).all()
    assert np.array_equal(got[~mask], base[~mask])
    if pad or shift:
        assert bool(around(y, rows, cols).isnan().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p,add", [(0.1, False), (0.5, True), (0.0, True), (0.999, False)])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 2048), (3, 7), (5, 8), (40, 129), (515, 2050), (1000, 64)])
def test_dropout(rows, cols, dtype, p, add):
    check(rows, cols, dtype, p, add)


@pytest.mark.parametrize("alias", [None, "x", "y_in"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(6, 40, 8, 8), (9, 5, 3, 1), (300, 131, 1, 3), (17, 1, 2, 0), (50, 16, 5, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views(rows, cols, pad, shift, alias, dtype):
    """The mask is that of the elements' places in the matrix, whatever the strides."""
    check(rows, cols, dtype, 0.3, True, pad, shift, alias)


@pytest.mark.parametrize("seed,offset,more", [(0, 0, None), (2 ** 64 - 1, 2 ** 64 - 1, None), (1, 2 ** 32 - 1, 1), (1 << 40, 2 ** 64 - 2, 5)])
def test_numbers_of_64_bits(seed, offset, more):
    check(33, 100, "f32", 0.25, False, seed=seed, offset=offset, more=more)


def test_the_share_of_what_is_dropped():
    """4 M elements: the share has a standard deviation of sqrt(p (1 - p) / 4e6); six of them."""
    x = torch.ones(1000, 4000, device=DEV)
    y = torch.empty_like(x)
    for p in (0.05, 0.5):
        dlcx.dlcx_dropout(x, None, y, p, 7, 1)
        assert abs(float((y == 0).float().mean()) - p) <= 6 * (p * (1 - p) / 4e6) ** 0.5 + 2.0 ** -17
        z = torch.empty_like(x)
        dlcx.dlcx_dropout(x, None, z, p, 7, 2)       # another offset: independent
        both = float(((y == 0) & (z == 0)).float().mean())
        assert abs(both - p * p) <= 6 * (p * p * (1 - p * p) / 4e6) ** 0.5 + 2.0 ** -16


def test_gradient_is_the_same_call():
    """dropout(x) . c is linear in x: its gradient is the same call on c, to the rounding of a product."""
    gen = torch.Generator().manual_seed(1)
    x, c = matrix(gen, 100, 333, torch.float32), matrix(gen, 100, 333, torch.float32)
    y, dx = torch.empty(100, 333, device=DEV), torch.empty(100, 333, device=DEV)
    dlcx.dlcx_dropout(x, None, y, 0.2, SEED, 3)
    dlcx.dlcx_dropout(c, None, dx, 0.2, SEED, 3)
    left, right = f64(y) * f64(c), f64(dx) * f64(x)
    assert (np.abs(left - right) <= 4 * U * np.abs(left)).all()
    z = x.clone()                                     # a difference: linear, so a step of any length
    z[40, 50:90] += 1.0
    moved = torch.empty_like(y)
    dlcx.dlcx_dropout(z, None, moved, 0.2, SEED, 3)
    rise = ((f64(moved) - f64(y)) * f64(c)).sum()
    slope = (f64(dx) * (f64(z) - f64(x))).sum()
    assert abs(rise - slope) <= 8 * U * (np.abs(f64(c)) * (np.abs(f64(moved)) + np.abs(f64(y)))).sum()


def test_values_that_are_dropped_do_not_count():
    x = torch.full((50, 60), float("nan"), device=DEV)
    y = torch.empty_like(x)
    dlcx.dlcx_dropout(x, None, y, 0.5, 1, 2)
    mask = torch.from_numpy(kept(3000, 0.5, 1, 2).reshape(50, 60)).to(DEV)
    assert bool(y[mask].isnan().all()) and not bool(y[~mask].any())


def test_a_captured_call_draws_anew():
    x, y = torch.ones(30, 700, device=DEV), torch.empty(30, 700, device=DEV)
    step = torch.zeros(1, device=DEV, dtype=torch.int64)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dlcx.dlcx_dropout(x, None, y, 0.4, 9, 100, step)
    for k in range(4):
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(f64(y) != 0, kept(21000, 0.4, 9, 100 + k).reshape(30, 700))
        step += 1
