"""Dropout of the rows that adapters read: in training only, and which projections and steps share a mask."""
import pytest
import torch

from eight_ref import DEV, TYPES, matrix
from paper_2506_21263_amd import inner

pytestmark = pytest.mark.gpu


def projection(dtype, base_bits, dropout, **kw):
    gen = torch.Generator().manual_seed(5)
    m, n, K, r = 72, 96, 2, 4
    theta = matrix(gen, m, n, torch.float32, 0.1)
    proj = inner.AdapterProjection(theta, torch.randn(K, r, n, generator=gen).to(DEV), 1.5, 40, TYPES[dtype], base_bits,
                                   dropout, **kw)
    p0 = torch.randn(K, r, m, generator=gen).to(DEV)
    proj.p.copy_(p0)
    if dtype == "bf16":
        proj.p_copy.copy_(p0)
    x, dy = matrix(gen, 40, n, TYPES[dtype]), matrix(gen, 40, m, TYPES[dtype])
    return proj, inner.Route((torch.arange(40) // 20).to(torch.int32).to(DEV), K), x, dy


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("base_bits", [8, 16])
def test_evaluation_drops_nothing(base_bits, dtype):
    """The same bits as a projection without dropout, both ways."""
    results = []
    for dropout in (0.3, 0.0):
        proj, route, x, dy = projection(dtype, base_bits, dropout)
        y, h = proj.forward(x, route, training=False)
        dx = proj.backward(x, h, dy, route, training=False)
        results.append([t.clone() for t in (y, h, dx, proj.dq, proj.dp)])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    proj, route, x, dy = projection(dtype, base_bits, 0.3)
    y, h = proj.forward(x, route, draw=1)
    assert not torch.equal(y, results[0][0])


def test_two_projections_have_masks_of_their_own():
    """Two of one shape, in the same step; with one seed they have one mask."""
    ys = []
    for kw in ({}, {}, dict(seed=3), dict(seed=3)):
        proj, route, x, _ = projection("f32", 16, 0.3, **kw)
        ys.append(proj.forward(x, route, draw=7)[0])
    assert not torch.equal(ys[0], ys[1]) and torch.equal(ys[2], ys[3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_captured_step_draws_anew(dtype):
    """A step with weights in 8 bits, whose number is on the device: replays have the masks of the numbers that it had,
    and the bits of eager steps with these numbers."""
    proj, route, x, dy = projection(dtype, 8, 0.3)
    step = torch.zeros(1, device=DEV, dtype=torch.int64)

    def both(draw):
        y, h = proj.forward(x, route, draw=draw)
        dx = proj.backward(x, h, dy, route, draw=draw)
        return y, h, dx, proj.dq, proj.dp

    both(step)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = both(step)
    seen = []
    for k in (0, 1, 2, 1 << 40):
        step.fill_(k)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = both(k)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        seen.append(got[0])
    assert not any(torch.equal(a, b) for a, b in zip(seen, seen[1:]))
