"""Inner steps and outer steps together: workers that train adapters beside one shared matrix."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV
from paper_2506_21263_amd import inner
from paper_2506_21263_amd.stage import MatrixState

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,dtype", [(32, torch.bfloat16), (8, torch.bfloat16), (32, torch.float32)], ids=str)
def test_workers_come_closer_to_their_teacher(bits, dtype):
    losses = inner.train(bits=bits, dtype=dtype)
    # nothing is applied after the first outer step (the one-step delay); from then on every average is
    assert abs(losses[1] - losses[0]) < 0.1 * losses[0]
    assert losses[-1] < 0.5 * losses[0], losses


def test_pseudo_gradients_of_adapters_are_those_of_their_replicas():
    gen = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=gen).to(DEV)  # noqa: E731
    m, n, K, r = 256, 320, 3, 12
    theta = 0.02 * rnd(m, n)
    M = MatrixState(theta.clone(), K, rnd(24, n), 8, 64, dlcx.MMA_F32)
    proj = inner.AdapterProjection(theta, rnd(K, r, n), 0.5, 64, torch.float32)
    proj.p.copy_(rnd(K, r, m))
    step = inner.AdapterOuterStep(M, 0.7, 0.9)
    p, q = proj.p.double(), proj.q.double()
    step.step(proj)
    for a in range(K):
        replica = theta.double() + 0.5 * torch.mm(p[a].t(), q[a])
        want = theta.double() - replica            # no error buffer yet
        got = M.ef[a].double()
        assert float((got - want).norm() / want.norm()) < 1e-5
    assert not proj.p.any() and torch.equal(M.theta_g, theta)   # outer step 1 applies nothing


def test_one_training_step_is_the_formulas():
    gen = torch.Generator().manual_seed(4)
    rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    m, n, K, r, rows = 96, 128, 2, 6, 50
    theta, q0, x = 0.1 * rnd(m, n), rnd(K, r, n) * 0.1, rnd(K * rows, n)
    p0, w = rnd(K, r, m) * 0.1, rnd(K * rows, m) * 0.01
    proj = inner.AdapterProjection(theta.to(DEV), q0.to(DEV), 2.0, K * rows, torch.float32)
    proj.p.copy_(p0)
    opts = [inner.AdamW(*proj.parameters(a)[:2], 1e-2, max_norm=0.05) for a in range(K)]
    route = inner.Route((torch.arange(K * rows) // rows).to(torch.int32).to(DEV), K)
    y, h = proj.forward(x.to(DEV), route)
    dx = proj.backward(x.to(DEV), h, w.to(DEV), route)
    for o in opts:
        o.step()
    for a in range(K):
        at = slice(a * rows, (a + 1) * rows)
        leaf = [t.double().requires_grad_() for t in (p0[a], q0[a], x[at])]
        out = leaf[2] @ (theta.double() + 2.0 * leaf[0].t() @ leaf[1]).t()
        (out * w[at].double()).sum().backward()
        close = lambda g, v: float((g.double().cpu() - v).norm() / v.norm()) < 1e-5  # noqa: E731
        assert close(y[at], out.detach()) and close(dx[at], leaf[2].grad)
        assert close(proj.dp[a], leaf[0].grad) and close(proj.dq[a], leaf[1].grad)
        norm = (leaf[0].grad.norm() ** 2 + leaf[1].grad.norm() ** 2).sqrt()
        assert abs(float(opts[a].norm) / float(norm) - 1) < 1e-5
        c = min(1.0, 0.05 / float(norm))
        for got, t, g in ((proj.p[a], p0[a], leaf[0].grad), (proj.q[a], q0[a], leaf[1].grad)):
            want = t.double() - 1e-2 * c * g / ((c * g).abs() + 1e-8)   # the first step of AdamW
            assert float((got.double().cpu() - want).abs().max()) < 1e-6
