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


def test_an_optimizer_made_on_one_stream_steps_on_another():
    gen = torch.Generator().manual_seed(7)
    start, grad = (torch.randn(50001, generator=gen).to(DEV) for _ in range(2))
    reference, buf = start.clone(), grad.clone()
    opt = inner.AdamW([reference], [buf], 1e-2, max_norm=0.5)
    for _ in range(3):
        opt.step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    param, buf = start.clone(), grad.clone()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)  # what follows on this stream is late
    opt = inner.AdamW([param], [buf], 1e-2, max_norm=0.5)
    opt.step(stream=streams[0])
    with torch.cuda.stream(streams[0]):
        torch.cuda._sleep(100_000_000)
    opt.step(stream=streams[1].cuda_stream)
    opt.step()
    assert torch.equal(param, reference) and opt.taken() == 3
    with torch.cuda.stream(streams[1]):
        torch.cuda._sleep(100_000_000)
        opt.step()
    opt.reset()
    assert not opt.moments[0]["m"].any() and not opt.moments[0]["v"].any()


@pytest.mark.parametrize("late", ["route", "use"])
def test_a_route_made_on_one_stream_serves_another(late):
    gen = torch.Generator().manual_seed(8)
    rnd = lambda *s: torch.randn(*s, generator=gen).to(DEV)  # noqa: E731
    m, n, K, r, rows = 128, 192, 3, 32, 700
    proj = inner.AdapterProjection(0.1 * rnd(m, n), rnd(K, r, n), 1.0, rows, torch.float32)
    proj.p.copy_(rnd(K, r, m))
    x, dy = rnd(rows, n), rnd(rows, m)
    ids = torch.randint(0, K, (rows,), generator=gen).to(torch.int32).to(DEV)
    route = inner.Route(ids, K)
    y, h = proj.forward(x, route)
    dx = proj.backward(x, h, dy, route)
    grads = proj.dq.clone(), proj.dp.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    if late == "route":
        with torch.cuda.stream(side):
            torch.cuda._sleep(200_000_000)
        route = inner.Route(ids, K, stream=side)
        y2, h2 = proj.forward(x, route)
        dx2 = proj.backward(x, h2, dy, route)
    else:
        torch.cuda._sleep(200_000_000)
        route = inner.Route(ids, K)
        with torch.cuda.stream(side):
            y2, h2 = proj.forward(x, route)
            dx2 = proj.backward(x, h2, dy, route)
        torch.cuda.current_stream().wait_stream(side)
    for a, b in zip((y, h, dx) + grads, (y2, h2, dx2, proj.dq, proj.dp)):
        assert torch.equal(a, b)


def test_steps_and_routes_are_captured_into_a_graph():
    gen = torch.Generator().manual_seed(9)
    rnd = lambda *s: torch.randn(*s, generator=gen).to(DEV)  # noqa: E731
    m, n, K, r, rows = 64, 64, 2, 32, 400
    proj = inner.AdapterProjection(0.1 * rnd(m, n), rnd(K, r, n), 1.0, rows, torch.float32)
    proj.p.copy_(rnd(K, r, m))
    route = inner.Route((torch.arange(rows, device=DEV) % K).to(torch.int32), K)
    x = rnd(rows, n)
    param, grad = rnd(5000), rnd(5000)
    opt = inner.AdamW([param], [grad], 1e-2, max_norm=0.5)
    first = param.clone()
    y, _ = proj.forward(x, route)
    opt.step()
    want = param.clone()
    graph = torch.cuda.CUDAGraph()
    opt.reset()
    with torch.cuda.graph(graph):
        y2, _ = proj.forward(x, route)
        opt.step()
    for _ in range(3):
        param.copy_(first)
        for t in opt.moments[0].values():
            t.zero_()
        y2.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(param, want) and torch.equal(y, y2)
    assert opt.taken() == 1


@pytest.mark.parametrize("bits,dtype", [(32, torch.float32), (8, torch.float32), (32, torch.bfloat16), (8, torch.bfloat16)],
                         ids=str)
@pytest.mark.parametrize("m,n,K,r", [(51, 35, 3, 5), (1021, 2050, 2, 33), (64, 66, 4, 1), (17, 19, 1, 3), (33, 37, 2, 255)])
def test_optimizers_of_adapters_of_any_size(m, n, K, r, bits, dtype):
    gen = torch.Generator().manual_seed(m)
    rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    rows = 40
    theta, q0, p0, x, dy = 0.1 * rnd(m, n), rnd(K, r, n) / n ** 0.5, rnd(K, r, m) * 0.1, rnd(K * rows, n), rnd(K * rows, m)
    proj = inner.AdapterProjection(theta.to(DEV), q0.to(DEV), 2.0, K * rows, dtype)
    proj.p.copy_(p0)
    proj.p_copy.copy_(p0)
    route = inner.Route((torch.arange(K * rows) // rows).to(torch.int32).to(DEV), K)
    opts = [inner.AdamW(*(lambda p, g, c: (p, g, 1e-2, (0.9, 0.95), 1e-8, None, c, bits))(*proj.parameters(a)))
            for a in range(K)]
    xd, dyd = x.to(DEV).to(dtype), dy.to(DEV).to(dtype)
    y, h = proj.forward(xd, route)
    dx = proj.backward(xd, h, dyd, route)
    for o in opts:
        o.step()
    # a few roundings to bf16 of operands and results, or sums of fp32
    tol = 2e-2 if dtype == torch.bfloat16 else 1e-5
    close = lambda g, v: float((g.double().cpu() - v).norm()) <= tol * float(v.norm())  # noqa: E731
    for a in range(K):
        at = slice(a * rows, (a + 1) * rows)
        p, q, w = p0[a].to(dtype).double(), q0[a].to(dtype).double(), theta.to(dtype).double() + 0
        xa, da = x[at].to(dtype).double(), dy[at].to(dtype).double()
        g = 2.0 * da @ p.t()
        assert close(y[at], xa @ w.t() + 2.0 * (xa @ q.t()) @ p) and close(dx[at], da @ w + g @ q)
        assert close(proj.dq[a], g.t() @ xa) and close(proj.dp[a], 2.0 * (xa @ q.t()).t() @ da)
        for master, copy, start, grad in ((proj.p[a], proj.p_copy[a], p0[a], proj.dp[a]), (proj.q[a], proj.q_copy[a], q0[a], proj.dq[a])):
            step = grad.double().cpu()
            want = start.double() - 1e-2 * step / (step.abs() + 1e-8)  # the first step of AdamW
            assert float((master.double().cpu() - want).abs().max()) < 2e-6
            assert torch.equal(copy, master.to(dtype))
    for t in proj.stored.values():
        assert not t[:, r:].any()  # nothing in the columns that are only stored


def test_a_step_is_captured_while_the_norm_of_the_last_one_is_on_its_way():
    gen = torch.Generator().manual_seed(10)
    start, grad = (torch.randn(5000, generator=gen).to(DEV) for _ in range(2))
    param, buf = start.clone(), grad.clone()
    opt = inner.AdamW([param], [buf], 1e-2, max_norm=0.5)
    for _ in range(3):
        opt.step()
    want = param.clone()
    param, buf = start.clone(), grad.clone()
    opt = inner.AdamW([param], [buf], 1e-2, max_norm=0.5)
    opt.step()
    assert opt.norm_there is not None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    graph.replay()
    opt.step()
    assert torch.equal(param, want) and opt.taken() == 3
