"""Outer steps of adapters whose rank is not the outer step's, and optimizers over their factors."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV
from paper_2506_21263_amd import inner
from paper_2506_21263_amd.stage import MatrixState

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mma", [dlcx.MMA_F32, dlcx.MMA_BF16, dlcx.MMA_FMA])
def test_adapters_of_a_higher_rank_than_the_outer_steps(mma):
    gen = torch.Generator().manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=gen).to(DEV)  # noqa: E731
    m, n, K, r = 256, 512, 2, 64
    theta = 0.02 * rnd(m, n)
    M = MatrixState(theta.clone(), K, rnd(8, n), 8, 64, mma)
    proj = inner.AdapterProjection(theta, rnd(K, r, n), 0.5, 64, torch.float32)
    step = inner.AdapterOuterStep(M, 0.7, 0.9)
    for _ in range(2):
        proj.p.copy_(rnd(K, r, m))
        p, q, e = proj.p.double(), proj.q.double(), [t.double() for t in M.ef]
        if step.t:  # what the delayed average takes out of the error buffer first
            d_hat = torch.mm(M.p_hat[:8].double().t(), M.q_bar[:8].double())
            e = [t - d_hat for t in e]
        step.step(proj)
        for a in range(K):
            want = e[a] - 0.5 * torch.mm(p[a].t(), q[a])
            # one fp32 sum of 64 products (two bf16 pieces: 2^-16 each)
            assert float((M.ef[a].double() - want).norm() / want.norm()) < (1e-5 if mma != dlcx.MMA_BF16 else 1e-4)
