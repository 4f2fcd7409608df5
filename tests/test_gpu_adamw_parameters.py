"""The parameter of a step with 8-bit moments: every operation on the way to it is one of fp32, rounded as fp32 rounds.

The chain is followed in numpy, operation by operation.  A root or a quotient that is off by more than half a unit in the
last place shows as another last bit of the update in a good part of the elements; 1e-4 units beyond the half, in one of
some thousands."""
import numpy as np
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV
from test_gpu_adamw import G, make, table_of, to_gpu

pytestmark = pytest.mark.gpu

F = np.float32
LR, B1, B2, STEP = 1e-2, 0.9, 0.95, 3


def chain(t, eps):
    """The updated parameter, from a parameter of zeros."""
    g = t["grad"].float().numpy()
    ms, vs = (t[k].repeat_interleave(G).numpy()[:g.size] for k in ("m_scale", "v_scale"))
    m, v = t["m"].float().numpy(), t["v"].float().numpy()
    with np.errstate(over="ignore", under="ignore", invalid="ignore"):
        m, v = m * np.abs(m) * ms, v * v * vs
        v = v * v
        m = m * F(B1) + g * F(1 - B1)
        v = v * F(B2) + g * g * F(1 - B2)
        inv = F(1 / np.sqrt(1 - B2 ** STEP))
        d = (np.sqrt(v).astype(np.float64) * float(inv) + float(F(eps))).astype(F)  # one rounding
        return -(m / d * F(LR / (1 - B1 ** STEP)))


@pytest.mark.parametrize("size,eps", [(1e-3, 1e-8), (1e-8, 1e-8), (1e-3, 1e-12), (1e6, 1e-8), (1e-18, 1e-25), (1e13, 1e-8)])
def test_updates_are_rounded_as_fp32_rounds(size, eps):
    t = make(1 << 18, torch.float32, torch.float32, 8, 3, size=size)
    t["param"] = torch.zeros(1 << 18)
    dev = to_gpu([t])[0]
    dlcx.dlcx_adamw(table_of([dev]), lr=LR, beta1=B1, beta2=B2, eps=eps, step=STEP)
    want, got = chain(t, eps), dev["param"].cpu().numpy()
    steps = np.abs(got.view(np.int32).astype(np.int64) - want.view(np.int32).astype(np.int64))
    assert np.isfinite(want).all() and (np.sign(got) == np.sign(want)).all()
    assert steps.max() <= 1 and np.mean(steps > 0) < 1e-3, (steps.max(), np.mean(steps > 0))


@pytest.mark.parametrize("gradient", [0.0, 1e-25, 3e19, 3e38, float("inf"), float("nan")])
def test_where_squares_leave_the_range(gradient):
    """v of zero, or below what fp32 holds, beyond it, and what is not a number: as the formula in fp32 has it."""
    t = make(2 * G, torch.float32, torch.float32, 8, 4)
    for k in ("m", "v", "m_scale", "v_scale", "param"):
        t[k] = torch.zeros_like(t[k])
    t["grad"][:G] = gradient
    dev = to_gpu([t])[0]
    dlcx.dlcx_adamw(table_of([dev]), lr=LR, beta1=B1, beta2=B2, eps=1e-8, step=STEP)
    want, got = chain(t, 1e-8), dev["param"].cpu().numpy()
    assert np.array_equal(np.isnan(want), np.isnan(got))
    fine = ~np.isnan(want)
    assert (np.abs(got[fine] - want[fine]) <= 2.0 ** -23 * np.abs(want[fine])).all()
