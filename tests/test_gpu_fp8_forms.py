"""Every kernel behind the product in 8 bits at sums of many blocks, against the same codes in 64 bits on the GPU.

Bounds: as in test_gpu_fp8.py for single outputs.  fp32 results are held to two more, which sums of the cores' 8-bit
products (1.5e-5 of a result) do not keep: sums whose every part fp32 holds come out exactly, and the error of many
outputs together.  A sum has at most n / 8 additions, each off by at most 2^-24 of a partial sum; partial sums of terms
with random signs are no larger in the mean square than the result, and the errors' signs are random, too, so together
they are at most sqrt(n / 8) 2^-24 of the results' root mean square."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from eight_forms import BF16, F32, FORMS, RING, TILES, WIDE
from eight_ref import DEV, HALF, TYPES, around, matrix

pytestmark = pytest.mark.gpu
CODE = {F32: dlcx.F32, BF16: dlcx.BF16}
IDS = ["%dx%dx%d-%s" % (*size, dtype) for size, dtype, _ in FORMS]


def values(a):
    """What a matrix stands for, in 64 bits."""
    codes, scales = a.held
    unit = (scales.view(torch.uint8).long() + (1023 - 127) << 52).view(torch.float64)   # (bytes from 1 on)
    return (codes.view(torch.float8_e4m3fn).double() * unit.repeat_interleave(128, 1)[:, :codes.shape[1]])[:, :a.cols]


def operand(gen, rows, cols):
    """Random codes (no NaN) and scales; the pad of the scales is 255."""
    a = dlcx.fp8_empty(rows, cols, DEV)
    codes, scales = (t.view(torch.uint8) for t in a.held)
    codes.zero_()
    c = torch.randint(0, 256, (rows, cols), generator=gen, device=DEV, dtype=torch.uint8)
    codes[:, :cols] = torch.where((c & 127) == 127, 0x38, c)
    scales.copy_(torch.randint(118, 128, scales.shape, generator=gen, device=DEV, dtype=torch.uint8))
    scales[:, -(-cols // 128):] = 255
    return a


def workspace(rows, m, n):
    return torch.empty(dlcx.dlcx_fp8_product_workspace_bytes(rows, m, n), device=DEV, dtype=torch.uint8).fill_(255)


@pytest.mark.parametrize("size,dtype,plan", FORMS, ids=IDS)
def test_values(size, dtype, plan):
    assert dlcx.dlcx_fp8_product_plan(*size, CODE[dtype]) == plan
    rows, m, n = size
    gen = torch.Generator(device=DEV).manual_seed(rows + 5 * m + 7 * n)
    x, w, ws, dt = operand(gen, rows, n), operand(gen, m, n), workspace(rows, m, n), TYPES[dtype]
    xv, wv = values(x), values(w)
    exact, most = xv @ wv.t(), xv.abs() @ wv.t().abs()
    for add in (False, True):                          # alone; then in place, rows apart, not aligned
        y = matrix(torch.Generator().manual_seed(1), rows, m, dt, 100.0, 3 * add, add)
        base = y.double() if add else torch.zeros((), device=DEV, dtype=torch.float64)
        want, size_of = exact + base, most + base.abs()
        dlcx.dlcx_fp8_product(x, w, y if add else None, y, ws)
        bound = (n + 8) * 2.0 ** -23 * size_of
        if dtype == BF16:
            bound += 2.0 ** -10 * size_of + HALF[dt] * want.abs() * 1.01
        assert bool(((y.double() - want).abs() <= bound).all())
        if add:
            assert bool(around(y, rows, m).isnan().all())


FP32 = [(size, plan) for size, dtype, plan in FORMS if dtype == F32]


@pytest.mark.parametrize("scale_x,scale_w", [(127, 127), (20, 234)])   # as codes are widened, and block by block
@pytest.mark.parametrize("size,plan", FP32, ids=[i for i, f in zip(IDS, FORMS) if f[1] == F32])
def test_exact_sums(size, plan, scale_x, scale_w):
    """Every eight terms have one of 2^8 or -2^8, which the eight beside them take away, and seven of 2^-6 to 2^-9.  Sums
    are multiples of 2^-9; within a block of 128 none passes 2^12, whatever the order, and those of whole blocks are below
    2^7, so fp32 holds all of them.  A cut at 2^-13 of the largest of eight would leave nothing."""
    rows, m, n = size
    x, w = dlcx.fp8_empty(rows, n, DEV), dlcx.fp8_empty(m, n, DEV)
    at = torch.arange(n)
    runs = n // 16 * 2                                 # (of eight; what is left at the end has small terms alone)
    small = torch.tensor([0x08, 0x04, 0x02, 0x01], dtype=torch.uint8)[(at // 8 + at) % 4]
    large = torch.where(at // 8 % 2 == 0, 0x78, 0xf8).to(torch.uint8)
    codes = torch.where((at % 8 == 3) & (at // 8 < runs), large, small)
    for a, c, s in ((x, codes.to(DEV), scale_x), (w, 0x38, scale_w)):
        a.held[0].view(torch.uint8).zero_()
        a.held[0].view(torch.uint8)[:, :n] = c
        a.held[1].fill_(s)
    x.held[0].view(torch.uint8)[rows - 1] ^= 128                       # the last row's signs are the others' turned round
    x.held[0].view(torch.uint8)[rows - 1, n:] = 0
    want = (values(x) @ values(w)[:1].t()).expand(rows, m)
    assert torch.equal(want, want.float().double()) and bool((want != 0).all())
    y = torch.empty(rows, m, device=DEV)
    dlcx.dlcx_fp8_product(x, w, None, y, workspace(rows, m, n))
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("size,plan", FP32, ids=[i for i, f in zip(IDS, FORMS) if f[1] == F32])
def test_error_of_many_outputs(size, plan):
    rows, m, n = size
    gen = torch.Generator(device=DEV).manual_seed(n)
    x, w = dlcx.fp8_empty(rows, n, DEV), dlcx.fp8_empty(m, n, DEV)
    for a in (x, w):
        dlcx.dlcx_fp8_quantize(torch.randn(a.rows, n, generator=gen, device=DEV), a)
    y = torch.empty(rows, m, device=DEV)
    dlcx.dlcx_fp8_product(x, w, None, y, workspace(rows, m, n))
    want = values(x) @ values(w).t()
    off = float((y.double() - want).square().mean().sqrt() / want.square().mean().sqrt())
    assert off <= (n / 8) ** 0.5 * 2.0 ** -24


@pytest.mark.parametrize("rows,m", [(3, 50), (40, 50), (300, 50), (1024, 1024)])
@pytest.mark.parametrize("n,scale", [(8192, 64), (128, 66), (1000, 60)])
def test_sums_of_the_smallest_products(rows, m, n, scale):
    """Products down to 2^-144 with scales that are applied as codes are widened (from 64 on), 2^-152 below them: sums that
    are numbers below fp32's normal range come out whole, or rounded where they end below 2^-149."""
    x, w = dlcx.fp8_empty(rows, n, DEV), dlcx.fp8_empty(m, n, DEV)
    for a in (x, w):
        a.held[0].view(torch.uint8).zero_()
        a.held[0].view(torch.uint8)[:, :n] = 1             # 2^-9
        a.held[1].fill_(scale)
    y = torch.empty(rows, m, device=DEV)
    dlcx.dlcx_fp8_product(x, w, None, y, workspace(rows, m, n))
    want = n * 2.0 ** (2 * (scale - 127 - 9))
    slack = 0.0 if scale >= 64 else -(-n // 128) * 2.0 ** -150     # half a step for every block that is added
    assert float((y.double() - want).abs().max()) <= slack


def test_same_bits_again_on_another_stream_and_from_a_graph():
    """One size of each kernel that the other such test leaves out: all of bf16, tiles of 256 x 256, and splits."""
    cases, seen = [], set()
    gen = torch.Generator(device=DEV).manual_seed(6)
    for (rows, m, n), dtype, plan in FORMS:
        kind = (dtype, plan[0], plan[1], plan[2] > 1)
        if kind in seen or (dtype == F32 and plan[0] not in (RING, TILES)) or rows * m > 1 << 23:
            continue
        seen.add(kind)
        x, w, dt = operand(gen, rows, n), operand(gen, m, n), TYPES[dtype]
        y_in = torch.randn(rows, m, generator=gen, device=DEV).to(dt)
        cases.append((x, w, y_in, torch.empty(rows, m, device=DEV, dtype=dt), workspace(rows, m, n)))
    assert (BF16, WIDE, 256, False) in seen and len(seen) > 15

    def run(stream=None):
        for x, w, y_in, y, ws in cases:
            dlcx.dlcx_fp8_product(x, w, y_in, y, ws, stream=stream)

    def check():
        torch.cuda.synchronize()
        assert all(torch.equal(c[3], v) for c, v in zip(cases, want))
        for _, _, _, y, ws in cases:
            y.zero_()
            ws.fill_(255)

    run()
    want = [c[3].clone() for c in cases]
    check()
    run()
    check()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    run(s)
    check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for _ in range(3):
        g.replay()
        check()
        run()                                              # eager work between the replays
        check()
