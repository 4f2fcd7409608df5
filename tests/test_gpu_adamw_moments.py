"""What nearest codes of 8 bits do to moments over many steps, at small and at usual rates of decay."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV
from test_gpu_adamw import G, moments, table_of

pytestmark = pytest.mark.gpu


def fresh(n):
    z = lambda k, dt=torch.float32: torch.zeros(k, device=DEV, dtype=dt)  # noqa: E731
    return dict(param=z(n), grad=z(n), m=z(n, torch.int8), v=z(n, torch.uint8), m_scale=z(-(-n // G)), v_scale=z(-(-n // G)))


@pytest.mark.parametrize("beta2,wide", [(0.95, 0.1), (0.99, 0.15), (0.999, 0.25)])
def test_moments_follow_gradients_that_keep_their_distribution(beta2, wide):
    # (the same recursion in numpy, other draws: nine of ten within 0.051, 0.10 and 0.18 after 4000 steps)
    n = 64 * G
    gen = torch.Generator(device=DEV).manual_seed(1)
    spread = torch.randn(n, generator=gen, device=DEV).exp()
    t = fresh(n)
    table = table_of([t])
    v = torch.zeros(n, device=DEV, dtype=torch.float64)
    for step in range(1, 1501):
        t["grad"].copy_(torch.randn(n, generator=gen, device=DEV) * spread)
        dlcx.dlcx_adamw(table, 1e-3, 0.9, beta2, 1e-8, step)
        v = beta2 * v + (1 - beta2) * t["grad"].double() ** 2
    ratio = (moments({k: x for k, x in t.items()})[1] / v).sqrt()
    low, mid, high = torch.quantile(ratio, torch.tensor([0.05, 0.5, 0.95], device=DEV, dtype=torch.float64)).tolist()
    assert 1 - wide < low and high < 1 + wide and abs(mid - 1) < wide / 4, (low, mid, high)


def stays(beta, power):
    """The codes that a decay without gradient leaves as they are: c beta^(1/power) rounds to c."""
    return [c for c in range(256) if c * (1 - beta ** (1 / power)) < 0.5]


@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.95), (0.9, 0.99), (0.9, 0.999), (0.5, 0.95)])
def test_where_a_moment_without_gradient_comes_to_rest(beta1, beta2):
    # one element of the group has the same gradient at every step, the others had theirs once
    t = fresh(G)
    t["m"][:] = torch.arange(G, device=DEV)
    t["v"][:] = (2 * torch.arange(G, device=DEV)).to(torch.uint8)
    t["m"][0], t["v"][0] = 127, 255
    t["m_scale"].fill_(1 / 127 ** 2)
    t["v_scale"].fill_(1 / 255 ** 2)
    t["grad"][0] = 1.0
    start_m, start_v = t["m"].clone().int(), t["v"].clone().int()
    table = table_of([t])
    for step in range(1, 2001):
        dlcx.dlcx_adamw(table, 0.0, beta1, beta2, 1e-8, step)
    assert t["m"][0] == 127 and t["v"][0] == 255
    last_m, last_v = stays(beta1, 2)[-1], stays(beta2, 4)[-1]
    assert torch.equal(t["m"][1:].int(), start_m[1:].clamp(max=min(last_m, 127)))
    assert torch.equal(t["v"][1:].int(), start_v[1:].clamp(max=min(last_v, 255)))
    if (beta1, beta2) == (0.9, 0.95):
        assert (last_m, last_v) == (9, 39)
    if beta2 == 0.999:
        assert torch.equal(t["v"][1:].int(), start_v[1:])  # no v falls


def test_a_usual_beta2_comes_down_too():
    # a badly scaled quadratic at beta2 = 0.999, as at 0.95
    n = 4096
    scale = torch.logspace(-2, 2, n).to(DEV)
    loss = {}
    for bits in (32, 8):
        t = fresh(n)
        if bits == 32:
            t = dict(param=t["param"], grad=t["grad"], m=torch.zeros(n, device=DEV), v=torch.zeros(n, device=DEV))
        t["param"].fill_(1.0)
        table = table_of([t])
        for step in range(1, 1001):
            t["grad"].copy_(scale * t["param"])
            dlcx.dlcx_adamw(table, 1e-2, 0.9, 0.999, 1e-8, step)
        loss[bits] = float((0.5 * scale * t["param"] ** 2).sum())
    start = float(0.5 * scale.sum())
    assert loss[32] < 1e-3 * start and loss[8] < 1e-2 * start, loss
