"""AdamW over many tensors, the gradients' norm and the 8-bit moments, against the formulas in 64 bits.

Bounds: the fp32 step makes a dozen operations of 2^-24 each on its way to a value; bf16 outputs add one
rounding of 2^-8.  A code of 8 bits is at most half a code from the root it stands for, and 1e-4 of a code
for the arithmetic that leads there (255 times a dozen roundings)."""
import math

import numpy as np
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = 2.0 ** -8
G = dlcx.STATE_GROUP
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8)


def make(numel, pdt, gdt, bits, seed, copy=False, decay=0.0, rate=1.0, size=1e-3):
    gen = torch.Generator().manual_seed(1000 * seed + numel)
    spread = torch.randn(-(-numel // 32), 1, generator=gen).exp().expand(-1, 32).reshape(-1)[:numel]
    t = dict(param=(torch.randn(numel, generator=gen) * 0.02).to(pdt),
             grad=(torch.randn(numel, generator=gen) * size * spread).to(gdt), weight_decay=decay, lr_scale=rate)
    m = torch.randn(numel, generator=gen) * size * spread
    v = (torch.randn(numel, generator=gen) * size * spread) ** 2
    if bits == 8:
        for name, x, top, dt in (("m", m, 127, torch.int8), ("v", v.sqrt(), 255, torch.uint8)):
            pad = torch.cat([x, x.new_zeros(-numel % G)]).view(-1, G)
            scale = pad.abs().amax(1) / top ** 2
            root = (pad.abs() / scale.clamp(min=1e-38)[:, None]).sqrt().round().clamp(max=top) * pad.sign()
            t[name], t[name + "_scale"] = root.view(-1)[:numel].to(dt), scale
    else:
        t["m"], t["v"] = m, v
    if copy:
        t["copy"] = torch.zeros(numel, dtype=torch.bfloat16)
    return t


def to_gpu(ts):
    return [{k: x.to(DEV) if isinstance(x, torch.Tensor) else x for k, x in t.items()} for t in ts]


def table_of(ts):
    memory = torch.empty(dlcx.dlcx_tensor_table_bytes(len(ts)), device=DEV, dtype=torch.uint8)
    return dlcx.dlcx_tensor_table([dlcx.tensor(**t) for t in ts], memory)


def moments(t):
    """m and v of a tensor in 64 bits."""
    if t["m"].dtype == torch.float32:
        return t["m"].double(), t["v"].double()
    n = t["m"].numel()
    ms, vs = (t[k].double().repeat_interleave(G)[:n] for k in ("m_scale", "v_scale"))
    m, v = t["m"].double(), t["v"].double()
    return m * m.abs() * ms, (v * v * vs) ** 2


def oracle(t, step, lr, beta1, beta2, eps, clip=1.0):
    g = t["grad"].double() * clip
    m, v = moments(t)
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    lr = lr * t["lr_scale"]
    move = lr / (1 - beta1 ** step) * m / ((v / (1 - beta2 ** step)).sqrt() + eps)
    p = t["param"].double() * (1 - lr * t["weight_decay"])
    return p - move, m, v, p.abs() + move.abs()


def check(before, after, step, clip=1.0, **hyper):
    for i, (t, got) in enumerate(zip(before, after)):
        got = {k: x.cpu() if isinstance(x, torch.Tensor) else x for k, x in got.items()}
        p, m, v, size = oracle(t, step, clip=clip, **{**HYPER, **hyper})
        n = p.numel()
        if n == 0:
            continue
        # m is a difference of magnitudes: bounded by theirs
        m_size = m.abs() + 2 * (1 - HYPER["beta1"]) * (t["grad"].double() * clip).abs()
        move = size - t["param"].double().abs()
        err = 16 * U * size + 16 * U * move.abs() * (m_size / m.abs().clamp(min=1e-300)).clamp(max=1e6)
        low = BF if t["param"].dtype == torch.bfloat16 else 0.0
        assert ((got["param"].double() - p).abs() <= err + low * p.abs() + 1e-30).all(), i
        if "copy" in t:
            assert torch.equal(got["copy"], got["param"].to(torch.bfloat16)), i
        if t["m"].dtype == torch.float32:
            assert ((got["m"].double() - m).abs() <= 8 * U * m_size).all(), i
            assert ((got["v"].double() - v).abs() <= 8 * U * v + 1e-44).all(), i
            continue
        for name, x, top, floor in (("m", m, 127, 0), ("v", v.sqrt(), 255, 1)):
            pad = torch.cat([x, x.new_zeros(-n % G)]).view(-1, G)
            scale = pad.abs().amax(1) / top ** 2
            there = got[name + "_scale"].double()
            assert ((there - scale).abs() <= 32 * U * scale).all(), (i, name)
            root = (pad.abs() / scale.clamp(min=1e-300)[:, None]).sqrt().view(-1)[:n]
            code = got[name].double()
            assert ((code.abs() - root).abs() <= 0.5 + 1e-4 + floor * 0.5 * (root < 0.5)).all(), (i, name)
            assert (code.abs() <= top).all() and (code[x.view(-1)[:n] > 0] >= floor).all(), (i, name)
            assert (code * x.view(-1)[:n] >= 0).all(), (i, name)


TYPES = [(p, g, b) for b in (32, 8) for p in (torch.float32, torch.bfloat16) for g in (torch.float32, torch.bfloat16)]


@pytest.mark.parametrize("pdt,gdt,bits", TYPES, ids=str)
def test_a_step_over_tensors_of_all_lengths(pdt, gdt, bits):
    lengths = [1, 7, 8, 9, 127, 128, 129, 0, 2047, 2048, 2049, 4095, 4096, 4097, 8192, 0, 100003, 3]
    ts = [make(n, pdt, gdt, bits, i, copy=pdt == torch.float32 and i % 2 == 0, decay=0.1 * (i % 3),
               rate=1.0 + 0.5 * (i % 2)) for i, n in enumerate(lengths)]
    dev = to_gpu(ts)
    dlcx.dlcx_adamw(table_of(dev), step=3, **HYPER)
    check(ts, dev, 3)


def test_tensors_of_all_types_in_one_table():
    ts = [make(50 + 977 * i, p, g, b, i, decay=0.01) for i, (p, g, b) in enumerate(TYPES * 3)]
    dev = to_gpu(ts)
    dlcx.dlcx_adamw(table_of(dev), step=1, **HYPER)
    check(ts, dev, 1)


@pytest.mark.parametrize("count", [64, 65, 4096, 4097, 9000])
def test_many_tensors_find_their_elements(count):
    sizes = [(7 * i) % 300 if i % 5 else 4096 + i % 3 for i in range(count)]
    flat = make(sum(-(-n // G) * G for n in sizes), torch.float32, torch.float32, 32, 5)
    views, at = [], 0
    dev = to_gpu([flat])[0]
    for i, n in enumerate(sizes):
        views.append({k: dev[k][at:at + n] for k in ("param", "grad", "m", "v")} | {"weight_decay": 0.1 * (i % 2)})
        at += -(-n // G) * G
    dlcx.dlcx_adamw(table_of(views), step=2, **HYPER)
    got = {k: dev[k].cpu() for k in ("param", "m", "v")}
    at = 0
    for i, n in enumerate(sizes):
        if i % 37 == 0 or i > count - 3:
            one = {k: flat[k][at:at + n] for k in ("param", "grad", "m", "v")} | {"lr_scale": 1.0, "weight_decay": 0.1 * (i % 2)}
            check([one], [{k: got[k][at:at + n] for k in got} | {"grad": one["grad"]}], 2)
        pad = slice(at + n, at + -(-n // G) * G)
        assert all(torch.equal(got[k][pad], flat[k][pad]) for k in got), i  # nothing beside a tensor is touched
        at += -(-n // G) * G


@pytest.mark.parametrize("bits", [32, 8])
def test_clipping_by_a_norm_on_the_device(bits):
    ts = [make(n, torch.float32, torch.float32, bits, i) for i, n in enumerate((300, 5000))]
    for norm, limit, clip in ((4.0, 1.0, 0.25), (0.5, 1.0, 1.0), (0.0, 1.0, 1.0), (1.0, 1.0, 1.0), (3.0, 0.3, 0.1)):
        dev = to_gpu(ts)
        dlcx.dlcx_adamw(table_of(dev), step=5, norm=torch.tensor([norm], device=DEV), max_norm=limit, grad_scale=0.5, **HYPER)
        check(ts, dev, 5, clip=0.5 * clip)
    for norm in (float("inf"), float("nan"), float("-inf")):  # the step is left out
        dev = to_gpu(ts)
        dlcx.dlcx_adamw(table_of(dev), step=5, norm=torch.tensor([norm], device=DEV), max_norm=1.0, **HYPER)
        for t, got in zip(ts, dev):
            assert all(torch.equal(got[k].cpu(), t[k]) for k in ("param", "m", "v"))


@pytest.mark.parametrize("gdt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lengths", [[1], [0], [0, 5], [4096], [33 * 1021, 1, 127], [1 << 22, 999, 4097]], ids=str)
def test_norm_of_the_gradients(gdt, lengths):
    ts = [make(n, torch.float32, gdt, 32, i) for i, n in enumerate(lengths)]
    dev = to_gpu(ts)
    table = table_of([{"grad": t["grad"]} for t in dev])
    out = torch.full((1,), -1.0, device=DEV)
    want = 0.25 * math.sqrt(sum(float((t["grad"].double() ** 2).sum()) for t in ts))
    for _ in range(3):  # the count of finished workgroups is back at 0 each time
        dlcx.dlcx_grad_norm(table, out, grad_scale=0.25)
        assert abs(float(out) - want) <= 2 * U * want
    if want > 0:
        with pytest.raises(dlcx.DlcxError):
            dlcx.dlcx_adamw(table, step=1, **HYPER)  # a table of gradients alone
    else:
        dlcx.dlcx_adamw(table, step=1, **HYPER)  # of no elements: there is nothing to do
    with pytest.raises(dlcx.DlcxError):
        dlcx.dlcx_grad_norm(table, out, grad_scale=float("nan"))


def test_norm_where_fp32_squares_would_not_do():
    for x in (1e25, 1e-30, 3e38):
        t = {"grad": torch.full((10007,), x, device=DEV)}
        out = torch.zeros(1, device=DEV)
        dlcx.dlcx_grad_norm(table_of([t]), out)
        want = float(torch.tensor(x).double()) * math.sqrt(10007.0)
        assert float(out) == want or abs(float(out) - want) <= 2 * U * want or want > 3.4e38 and math.isinf(float(out))
    for x in (float("inf"), float("nan")):
        t = {"grad": torch.ones(10007, device=DEV)}
        t["grad"][9999] = x
        dlcx.dlcx_grad_norm(table_of([t]), out)
        assert not math.isfinite(float(out))


def test_moments_of_8_bits_at_their_edges():
    # zeros, a group of one huge and many tiny values, values below what a group of 2^-100 keeps, a NaN
    n = 5 * G
    t = make(n, torch.float32, torch.float32, 8, 1)
    for k in ("m", "v", "m_scale", "v_scale"):
        t[k] = torch.zeros_like(t[k])
    g = torch.zeros(n)
    g[G] = 1e3
    g[G + 1:2 * G] = 1e-6
    g[2 * G:3 * G] = 1e-32
    g[3 * G:4 * G] = 0.5
    g[3 * G + 7] = float("nan")
    g[4 * G:] = -2.0
    t["grad"] = g
    dev = to_gpu([t])[0]
    dlcx.dlcx_adamw(table_of([dev]), step=1, **HYPER)
    m, v = dev["m"].cpu(), dev["v"].cpu()
    assert not m[:G].any() and not v[:G].any() and dev["m_scale"][0] == 0
    assert m[G] == 127 and v[G] == 255 and (v[G + 1:2 * G] == 1).all()   # tiny, and still no zero denominator
    assert not m[2 * G:3 * G].any() and dev["m_scale"][2] == 0
    assert torch.isnan(dev["m_scale"][3]) and torch.isnan(dev["v_scale"][3])  # a group keeps its NaN
    assert (m[4 * G:] == -127).all() and (v[4 * G:] == 255).all()
    keep = torch.ones(n, dtype=torch.bool)
    keep[3 * G + 7] = False
    assert torch.isfinite(dev["param"].cpu()[keep]).all()


@pytest.mark.parametrize("size", [1e-3, 1e-15, 1e-18, 1e12])
def test_codes_are_those_of_the_formula_to_the_last(size):
    """Every operation on the way to a code is one of fp32, rounded correctly: the codes of a step are those of
    the formula, also where a root is next to the middle of two of them (among 2^20 some hundreds are).
    (The roots here are numpy's: torch's on the CPU is not always the one next to the true root.)"""
    def root(x):
        return torch.from_numpy(np.sqrt(x.numpy()))

    t = make(1 << 20, torch.bfloat16, torch.bfloat16, 8, 5, size=size)
    dev = to_gpu([t])[0]
    dlcx.dlcx_adamw(table_of([dev]), step=2, **HYPER)
    g = t["grad"].float()
    ms, vs = (t[k].repeat_interleave(G) for k in ("m_scale", "v_scale"))
    m, v = t["m"].float(), t["v"].float()
    m, v = m * m.abs() * ms, v * v * vs
    m = m * HYPER["beta1"] + g * (1 - HYPER["beta1"])
    v = v * v * HYPER["beta2"] + g * g * (1 - HYPER["beta2"])
    for name, x, top, least in (("m", m, 127, 0), ("v", root(v), 255, 1)):
        scale = x.abs().view(-1, G).amax(1) * (1.0 / top ** 2)
        code = root(x.abs() / scale.repeat_interleave(G)).round().clamp(min=least) * x.sign()
        assert torch.equal(dev[name + "_scale"].cpu(), scale), name
        assert torch.equal(dev[name].cpu().float(), code), (name, (dev[name].cpu().float() != code).sum())


@pytest.mark.parametrize("second", [False, True])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_what_8_bit_moments_stand_for(second, out):
    t = make(3 * G + 5, torch.float32, torch.float32, 8, 4)
    name = "v" if second else "m"
    got = torch.empty(t["m"].numel(), device=DEV, dtype=out)
    dlcx.dlcx_state_decode(t[name].to(DEV), t[name + "_scale"].to(DEV), got)
    want = moments(t)[1 if second else 0]
    assert ((got.double().cpu() - want).abs() <= (4 * U + (BF if out == torch.bfloat16 else 0)) * want.abs()).all()


def test_8_bit_moments_lead_where_32_bits_lead():
    # a badly scaled quadratic: both forms come down, and to the same size (8-bit moments are not the same path)
    n = 4096
    scale = torch.logspace(-2, 2, n).to(DEV)
    loss = {}
    for bits in (32, 8):
        t = make(n, torch.float32, torch.float32, bits, 9)
        t["param"] = torch.ones(n)
        for k in ("m", "v") + (("m_scale", "v_scale") if bits == 8 else ()):
            t[k] = torch.zeros_like(t[k])
        dev = to_gpu([t])[0]
        table = table_of([dev])
        for step in range(1, 301):
            dev["grad"].copy_(scale * dev["param"])
            dlcx.dlcx_adamw(table, step=step, **HYPER)
        loss[bits] = float((0.5 * scale * dev["param"] ** 2).sum())
    start = float(0.5 * scale.sum())
    assert loss[32] < 1e-3 * start and loss[8] < 1e-3 * start, loss


def test_the_same_bits_on_another_stream_and_from_a_graph():
    ts = [make(n, p, g, b, i) for i, ((p, g, b), n) in enumerate(zip(TYPES, (1000, 5000, 129, 70000, 4096, 3, 999, 12345)))]
    ref = to_gpu(ts)
    norm = torch.zeros(1, device=DEV)

    def two_steps(dev, table):
        for step in (1, 2):
            dlcx.dlcx_grad_norm(table, norm)
            dlcx.dlcx_adamw(table, step=step, norm=norm, max_norm=0.05, **HYPER)

    two_steps(ref, table_of(ref))
    torch.cuda.synchronize()
    other = to_gpu(ts)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two_steps(other, table_of(other))
    side.synchronize()
    third = to_gpu(ts)
    table = table_of(third)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two_steps(third, table)
    keys = ("param", "m", "v")
    for _ in range(3):
        for t, src in zip(third, to_gpu(ts)):
            for k in src:
                if isinstance(src[k], torch.Tensor):
                    t[k].copy_(src[k])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(ref, other, third):
            assert all(torch.equal(a[k], b[k]) and torch.equal(a[k], c[k]) for k in keys)


def test_more_than_2_to_the_31_elements():
    n = (1 << 31) + 4097
    grad = torch.empty(n, device=DEV, dtype=torch.bfloat16).fill_(0.5)
    param = torch.empty(n, device=DEV, dtype=torch.bfloat16).fill_(1.0)
    m, v = torch.zeros(n, device=DEV, dtype=torch.int8), torch.zeros(n, device=DEV, dtype=torch.uint8)
    scales = [torch.zeros(-(-n // G), device=DEV) for _ in range(2)]
    table = table_of([dict(param=param, grad=grad, m=m, v=v, m_scale=scales[0], v_scale=scales[1])])
    out = torch.zeros(1, device=DEV)
    dlcx.dlcx_grad_norm(table, out)
    assert abs(float(out) - 0.5 * math.sqrt(n)) <= 2 * U * 0.5 * math.sqrt(n)
    dlcx.dlcx_adamw(table, step=1, **HYPER)
    for at in (0, 1 << 30, (1 << 31) - 1, 1 << 31, n - 1):
        assert m[at] == 127 and v[at] == 255 and abs(float(param[at]) - 0.99) < 0.99 * BF * 2
    assert int(m[-5000:].double().sum()) == 127 * 5000


def test_wrong_tensors_are_refused():
    t = to_gpu([make(300, torch.float32, torch.float32, 8, 1)])[0]
    for bad in (dict(grad=t["grad"].cpu()), dict(m=t["m"][:299]), dict(v=t["v"].to(torch.int8)), dict(param=t["param"][:200]),
                dict(m_scale=None), dict(v_scale=t["v_scale"][:2]), dict(copy=t["param"]), dict(grad=t["grad"][::2])):
        with pytest.raises((ValueError, dlcx.DlcxError)):
            table_of([{**t, **bad}])
    off = torch.zeros(301, device=DEV)[1:]
    with pytest.raises(dlcx.DlcxError):
        table_of([{**t, "grad": off}])  # not at 16 bytes
    table = table_of([t])
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(lr=float("nan")), dict(grad_scale=-1.0)):
        with pytest.raises(dlcx.DlcxError):
            dlcx.dlcx_adamw(table, **{**HYPER, "step": 1, **bad})
    with pytest.raises(dlcx.DlcxError):
        dlcx.dlcx_adamw(table, step=1, norm=torch.ones(1, device=DEV), max_norm=0.0, **HYPER)
