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


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("how", ["current", "stream", "handle"])
def test_a_step_that_is_left_out_does_not_count(bits, how):
    gen = torch.Generator().manual_seed(6)
    start = [torch.randn(s, generator=gen).to(DEV) for s in (300, 4097)]
    grads = [[torch.randn(p.shape, generator=gen).to(DEV) for p in start] for _ in range(4)]

    def run(steps):
        params, bufs = [p.clone() for p in start], [torch.empty_like(p) for p in start]
        opt = inner.AdamW(params, bufs, 1e-2, bits=bits, max_norm=0.5)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        for k in steps:
            with torch.cuda.stream(torch.cuda.current_stream() if how == "current" else side):
                for b, g in zip(bufs, grads[k] if k >= 0 else grads[0]):
                    b.copy_(g)
                if k < 0:
                    bufs[1][17] = float("inf") if k == -1 else float("nan")
            opt.step(stream=None if how == "current" else side if how == "stream" else side.cuda_stream)
        side.synchronize()
        return opt, params + [x for m in opt.moments for x in m.values()]

    plain, want = run([0, 1, 2, 3])
    opt, got = run([0, -1, 1, 2, -1, -2, 3])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert plain.taken() == 4 and opt.taken() == 4 and opt.taken() == 4
    opt, _ = run([0, 1, -1])
    assert opt.taken() == 2
    opt.reset()
    assert opt.taken() == 0
