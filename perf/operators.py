"""Performance cases of the inner step: what runs between two outer steps of a stage, while K workers
train low-rank adapters beside the shared projections, or requests are answered with them.

Sizes are those of the benchmark configurations (a 512 x 512 matrix, the matrices of an OPT-1.3B-like
layer and of a ~100B dense layer, ranks 8 .. 64, four workers) and odd sizes around them.  A case is
a dict of plain values whose "op" names the call:

  forward   dlcx_adapter_forward: y = y_in + s_a (x Q_a^T) P_a with the adapter a of each row
  backward  dlcx_adapter_backward: dx, dQ and dP of the same
  norm      dlcx_grad_norm: the global norm of the gradients of many tensors
  adamw     dlcx_adamw: an AdamW step over many tensors, states in 32 or in 8 bits; the latter are
            returned as the values that they stand for (dlcx_state_decode), in bf16: a code has
            no more than 8 significant bits

All inputs are drawn on the GPU from the seed: activations N(0, 1), factors and weights N(0, 0.02^2),
gradients and optimizer states with a scale that varies from one group of 128 elements to the next.
The tensors of a step are views of one buffer, each padded with zeros to a multiple of 128 elements,
so that the plain form works on the buffer as a whole.
"""
import math

import torch

own = False

DEV = "cuda"
GROUP = 128                          # elements that share a scale of the 8-bit states
BETA1, BETA2, EPS = 0.9, 0.95, 1e-8
LR, DECAY, STEP = 3e-4, 0.1, 200     # STEP: the step number that the first pass has
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
DENSE = "8192x8192*2,8192x1024*2,8192x28672*2,28672x8192"   # one layer of the ~100B dense stage
OPT = "2048x2048*4,2048x8192,8192x2048"                     # one OPT-1.3B-like layer
# factors (P: r x m, Q: r x n) of adapters of rank 16 beside every matrix of a ten-layer dense stage
FACTORS = "16x8192*90,16x1024*20,16x28672*30"


def listed():
    return [
        # one token of one request beside an OPT-1.3B projection: launches and latency count
        dict(name="forward-1-row-2048x2048-r8", op="forward", rows=1, m=2048, n=2048, r=8, count=4,
             dtype="bf16", order="mixed", ranks=False),
        # one token of each of 96 requests, 64 adapters of two ranks, some requests without any
        dict(name="forward-96-rows-28672x8192-r16", op="forward", rows=96, m=28672, n=8192, r=16,
             count=64, dtype="bf16", order="mixed", ranks=True),
        # the prompts of a dozen requests, of ragged lengths, one after the other
        dict(name="forward-4133-rows-8192x8192-r64", op="forward", rows=4133, m=8192, n=8192, r=64,
             count=12, dtype="bf16", order="requests", ranks=False),
        # odd sizes that no 16-byte access fits, fp32, rows of three adapters in any order
        dict(name="forward-1000-rows-1021x2050-r33", op="forward", rows=1000, m=1021, n=2050, r=33,
             count=3, dtype="f32", order="mixed", ranks=False),
        # a micro-batch of each of four workers beside the dense layer's projection: training
        dict(name="backward-16384-rows-8192x8192-r64", op="backward", rows=16384, m=8192, n=8192,
             r=64, count=4, dtype="bf16", order="workers", ranks=False),
        # a short ragged batch in fp32 beside an OPT-1.3B projection
        dict(name="backward-515-rows-2048x8192-r20", op="backward", rows=515, m=2048, n=8192, r=20,
             count=4, dtype="f32", order="requests", ranks=True),
        # 140 factor gradients of a stage's adapters
        dict(name="norm-stage-adapters-r16", op="norm", shapes=FACTORS, grad="f32"),
        # all gradients of a dense layer
        dict(name="norm-dense-layer-bf16", op="norm", shapes=DENSE, grad="bf16"),
        # the adapters of a stage: fp32 factors, and the bf16 copies that the products read
        dict(name="adamw32-stage-adapters-r16", op="adamw", shapes=FACTORS, vectors="", param="f32",
             grad="f32", bits=32, copy=True, clip=True),
        # an OPT-1.3B layer with its norms and biases (no decay): fp32 masters, bf16 gradients
        dict(name="adamw32-opt-layer", op="adamw", shapes=OPT, vectors="2048*9,8192", param="f32",
             grad="bf16", bits=32, copy=True, clip=False),
        # a whole dense layer, 8-bit states, bf16 weights
        dict(name="adamw8-dense-layer-bf16", op="adamw", shapes=DENSE, vectors="8192*2",
             param="bf16", grad="bf16", bits=8, copy=False, clip=True),
        # a few small tensors of odd lengths, 8-bit states: launches and latency count
        dict(name="adamw8-small-odd", op="adamw", shapes="512x512,33x1021", vectors="1,127,129,1021",
             param="f32", grad="f32", bits=8, copy=True, clip=False),
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    op = rng.choice(("forward", "forward", "forward", "backward", "backward", "norm", "adamw", "adamw", "adamw"))
    if op in ("forward", "backward"):
        dtype = rng.choice(("bf16", "bf16", "f32"))
        side = lambda: _log(rng, 256, 12000) if rng.random() < 0.3 else 16 * _log(rng, 16, 750)  # noqa: E731
        rows = _log(rng, 1 if op == "forward" else 16, 8192 if dtype == "bf16" else 2048)
        return dict(op=op, rows=rows, m=side(), n=side(), r=_log(rng, 1, 128), count=_log(rng, 1, 64),
                    dtype=dtype, order=rng.choice(("mixed", "requests", "workers")), ranks=rng.random() < 0.5)
    shapes = ",".join("%dx%d*%d" % (_log(rng, 1, 6000), _log(rng, 64, 6000), _log(rng, 1, 12))
                      for _ in range(rng.randint(1, 4)))
    grad = rng.choice(("f32", "bf16"))
    if op == "norm":
        return dict(op=op, shapes=shapes, grad=grad)
    param = rng.choice(("f32", "bf16"))
    return dict(op=op, shapes=shapes, vectors="%d*%d,%d" % (_log(rng, 1, 9000), _log(rng, 1, 30), _log(rng, 1, 9000)),
                param=param, grad=grad, bits=rng.choice((8, 32)), copy=param == "f32" and rng.random() < 0.5,
                clip=rng.random() < 0.5)


# ---- what a case's tensors are ----------------------------------------------------------------
def _lengths(text):
    """ "16x8192*3,7" -> [131072] * 3 + [7]"""
    out = []
    for part in text.split(","):
        if part:
            dims, _, times = part.partition("*")
            out += [math.prod(map(int, dims.split("x")))] * int(times or 1)
    return out


def _places(lengths, start=0):
    """Where each tensor begins in the common buffer, and where the last one's padding ends."""
    at = []
    for numel in lengths:
        at.append(start)
        start += -(-numel // GROUP) * GROUP
    return at, start


def _ranks(case):
    """Every other adapter has half the rank where a case has two of them."""
    r, half = case["r"], -(-case["r"] // 2)
    return [half if case["ranks"] and a % 2 else r for a in range(case["count"])]


def work(case):
    if case["op"] in ("forward", "backward"):
        rows, m, n, count = (case[k] for k in ("rows", "m", "n", "count"))
        size = TYPES[case["dtype"]].itemsize
        rank = sum(_ranks(case)) / count
        factors = min(rows, count) * rank * (m + n) * size
        if case["op"] == "forward":   # x, y_in, y, h, the factors in use
            return {"bytes": rows * (n + 2 * m) * size + rows * rank * 4 + factors, "flops": 2 * rows * rank * (m + n)}
        # x, dy, dx_in, dx, h, the factors in use, both gradients
        return {"bytes": rows * (3 * n + m) * size + rows * rank * 4 + factors + count * case["r"] * (m + n) * 4,
                "flops": 4 * rows * rank * (m + n)}
    grad = TYPES[case["grad"]].itemsize
    if case["op"] == "norm":
        numel = sum(_lengths(case["shapes"]))
        return {"bytes": numel * grad, "flops": 2 * numel}
    numel = sum(_lengths(case["shapes"])) + sum(_lengths(case["vectors"]))
    state = 16 if case["bits"] == 32 else 4 + 16 / GROUP + 4   # the last 4: both values, returned
    each = 2 * TYPES[case["param"]].itemsize + grad + state + (2 if case["copy"] else 0)
    return {"bytes": numel * each, "flops": 20 * numel}


# ---- inputs -----------------------------------------------------------------------------------
def _ids(case, gen):
    rows, count = case["rows"], case["count"]
    if case["order"] == "workers":        # equal shares, one after the other
        return (torch.arange(rows, device=DEV) * count // rows).to(torch.int32)
    draws = torch.rand(rows, generator=gen, device=DEV)
    if case["order"] == "requests":       # ragged shares, one after the other
        cuts = draws[: min(rows, count - 1)].sort().values * rows
        return torch.searchsorted(cuts, torch.arange(rows, device=DEV, dtype=torch.float32), right=True).to(torch.int32)
    ids = (draws * count).to(torch.int32).clamp_(max=count - 1)
    return torch.where((draws * 7919) % 1 < 0.05, -1, ids) if rows > 1 else ids   # one row in twenty without


def _prepare_adapter(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rows, m, n, r, count = (case[k] for k in ("rows", "m", "n", "r", "count"))
    dt = TYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(shape, generator=gen, device=DEV) * std).to(dtype)

    s = dict(case=case, x=normal(rows, n), ids=_ids(case, gen), q=normal(count, r, n, std=0.02),
             p=normal(count, r, m, std=0.02), scale=torch.rand(count, generator=gen, device=DEV) + 0.5,
             ranks=torch.tensor(_ranks(case), device=DEV, dtype=torch.int32) if case["ranks"] else None,
             out=torch.empty(rows, m if case["op"] == "forward" else n, device=DEV, dtype=dt),
             h=torch.empty(rows, r, device=DEV))
    if case["op"] == "forward":
        s["y_in"] = normal(rows, m)
    else:
        s["dy"], s["dx_in"] = normal(rows, m, std=1e-3), normal(rows, n, std=1e-3)
        s["h"] = (s["x"].float() @ s["q"].float().view(count * r, n).t()).mul_(_mask(s)).view(rows, count, r).sum(1)
        s["dq"], s["dp"] = torch.empty(count, r, n, device=DEV), torch.empty(count, r, m, device=DEV)
    if own:   # the workspace that a program keeps
        import paper_2506_21263_amd as dlcx
        s["desc"] = dlcx.adapter_desc(m, n, r, count, dlcx.BF16 if dt == torch.bfloat16 else dlcx.F32)
        s["workspace"] = torch.empty(dlcx.dlcx_adapter_workspace_bytes(s["desc"], rows), device=DEV, dtype=torch.uint8)
    return s


def _encode(x, top):
    """Codes and scales of groups of non-negative values: x = code^2 scale, the largest at code `top`."""
    x = x.view(-1, GROUP)
    scale = x.amax(1, keepdim=True) * (1.0 / (top * top))
    code = (x / scale).sqrt().round().clamp(max=top)
    return torch.where(scale > 0, code, 0.0), scale


def _prepare_tensors(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    first, rest = _lengths(case["shapes"]), _lengths(case.get("vectors", ""))
    at, decayed = _places(first)
    at2, total = _places(rest, decayed)
    lengths, at = first + rest, at + at2
    inside = torch.zeros(total, device=DEV, dtype=torch.bool)
    for a, numel in zip(at, lengths):
        inside[a:a + numel] = True

    def normal(std, spread=0.0):
        x = torch.randn(total // GROUP, GROUP, generator=gen, device=DEV).mul_(std)
        if spread:
            x.mul_((torch.randn(total // GROUP, 1, generator=gen, device=DEV) * spread).exp_())
        return x.view(-1).mul_(inside)

    s = dict(case=case, step=STEP, decayed=decayed, grad=normal(1e-3, 1.0).to(TYPES[case["grad"]]))
    views = [dict() for _ in lengths]
    s["norm"] = torch.zeros((), device=DEV)
    if case["op"] == "adamw":
        s["param"] = normal(0.02).to(TYPES[case["param"]])
        m, v = normal(3e-4, 1.0), normal(1e-3, 1.0).square_()
        if case["bits"] == 8:
            code, scale = _encode(m.abs(), 127)
            s["m"] = torch.where(m.view(-1, GROUP) < 0, -code, code).to(torch.int8).view(-1)
            s["m_scale"] = scale.view(-1)
            code, scale = _encode(v.sqrt_(), 255)
            s["v"] = torch.where(v.view(-1, GROUP) > 0, code.clamp(min=1), code).to(torch.uint8).view(-1)
            s["v_scale"] = scale.view(-1)
        else:
            s["m"], s["v"] = m, v
        if case["copy"]:
            s["copy"] = s["param"].to(torch.bfloat16)
        # the norm of all gradients of a model, of which a stage holds a part; twice the limit, or half
        s["norm"].fill_(2.0 if case["clip"] else 0.5)
        s["limit"] = torch.ones((), device=DEV)
        if case["bits"] == 8:
            s["m_value"], s["v_value"] = (torch.empty(total, device=DEV, dtype=torch.bfloat16) for _ in "mv")
        for view, a, numel in zip(views, at, lengths):
            view.update({k: s[k][a:a + numel] for k in ("param", "m", "v", "copy") if k in s})
            if case["bits"] == 8:
                view.update({k: s[k][a // GROUP:-(-(a + numel) // GROUP)] for k in ("m_scale", "v_scale")})
    for view, a, numel in zip(views, at, lengths):
        view["grad"] = s["grad"][a:a + numel]
        if case["op"] == "adamw":
            view["weight_decay"] = DECAY if a < decayed else 0.0
    if own:   # the table of its tensors that a program keeps
        import paper_2506_21263_amd as dlcx
        memory = torch.empty(dlcx.dlcx_tensor_table_bytes(len(views)), device=DEV, dtype=torch.uint8)
        s["views"], s["table"] = views, dlcx.dlcx_tensor_table([dlcx.tensor(**v) for v in views], memory)
    return s


def prepare(case, seed):
    return (_prepare_adapter if case["op"] in ("forward", "backward") else _prepare_tensors)(case, seed)


# ---- the operators ----------------------------------------------------------------------------
def _mask(s):
    """rows x (count r): one where the row has that adapter and the adapter that column."""
    count, r = s["case"]["count"], s["case"]["r"]
    mask = s["ids"][:, None] == torch.arange(count, device=DEV)
    mask = mask[:, :, None].expand(-1, -1, r)
    if s["ranks"] is not None:
        mask = mask & (torch.arange(r, device=DEV) < s["ranks"][:, None])
    return mask.reshape(-1, count * r).float()


def _plain_adapter(s):
    case = s["case"]
    rows, r, count, dt = case["rows"], case["r"], case["count"], TYPES[case["dtype"]]
    q, p = (s[k].float().view(count * r, -1) for k in "qp")
    mask = _mask(s)
    scaled = mask * s["scale"].repeat_interleave(r)
    x = s["x"].float()
    if case["op"] == "forward":
        h = x @ q.t()
        y = s["y_in"].float() + (h * scaled) @ p
        return {"y": y.to(dt), "h": (h * mask).view(rows, count, r).sum(1)}
    dy = s["dy"].float()
    g = (dy @ p.t()) * scaled
    h = s["h"].repeat(1, count) * scaled
    return {"dx": (s["dx_in"].float() + g @ q).to(dt), "dq": (g.t() @ x).view(count, r, -1),
            "dp": (h.t() @ dy).view(count, r, -1)}


def _values(s):
    """The states of an AdamW step as what they stand for."""
    if s["case"]["bits"] == 32:
        return s["m"], s["v"]
    c = s["m"].view(-1, GROUP).float()
    m = c * c.abs() * s["m_scale"][:, None]
    c = s["v"].view(-1, GROUP).float()
    return m.view(-1), (c * c * s["v_scale"][:, None]).square_().view(-1)


def _plain_adamw(s):
    case, t = s["case"], s["step"]
    g = s["grad"].float() * torch.where(s["norm"] > s["limit"], s["limit"] / s["norm"], 1.0)
    m, v = _values(s)
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    update = m / (v.sqrt() * (1.0 / math.sqrt(1.0 - BETA2 ** t)) + EPS) * (LR / (1.0 - BETA1 ** t))
    p, n = s["param"].float(), s["decayed"]
    p[:n] *= 1.0 - LR * DECAY
    p -= update
    s["param"].copy_(p)
    if case["copy"]:
        s["copy"].copy_(p)
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return
    code, scale = _encode(m.abs(), 127)
    s["m"].copy_(torch.where(m.view(-1, GROUP) < 0, -code, code).view(-1))
    s["m_scale"].copy_(scale.view(-1))
    code, scale = _encode(v.sqrt(), 255)
    s["v"].copy_(torch.where(v.view(-1, GROUP) > 0, code.clamp(min=1), code).view(-1))
    s["v_scale"].copy_(scale.view(-1))


def run(s):
    case = s["case"]
    if case["op"] == "norm":
        if not own:
            return {"norm": s["grad"].float().square().sum().sqrt()}
        import paper_2506_21263_amd as dlcx
        dlcx.dlcx_grad_norm(s["table"], s["norm"])
        return {"norm": s["norm"]}
    if case["op"] == "adamw":
        if own:
            import paper_2506_21263_amd as dlcx
            dlcx.dlcx_adamw(s["table"], LR, BETA1, BETA2, EPS, s["step"], norm=s["norm"], max_norm=1.0)
        else:
            _plain_adamw(s)
        s["step"] += 1
        out = {k: s[k] for k in ("param", "copy", "m_scale", "v_scale") if k in s}
        if case["bits"] == 32:
            return dict(out, m=s["m"], v=s["v"])
        if own:
            dlcx.dlcx_state_decode(s["m"], s["m_scale"], s["m_value"])
            dlcx.dlcx_state_decode(s["v"], s["v_scale"], s["v_value"])
            return dict(out, m=s["m_value"], v=s["v_value"])
        m, v = _values(s)
        return dict(out, m=m.to(torch.bfloat16), v=v.to(torch.bfloat16))
    if not own:
        return _plain_adapter(s)
    import paper_2506_21263_amd as dlcx
    if case["op"] == "forward":
        dlcx.dlcx_adapter_forward(s["desc"], s["x"], s["ids"], s["q"], s["p"], s["y_in"], s["out"], s["h"],
                                  s["workspace"], scale=s["scale"], ranks=s["ranks"])
        return {"y": s["out"], "h": s["h"]}
    dlcx.dlcx_adapter_backward(s["desc"], s["x"], s["dy"], s["ids"], s["q"], s["p"], s["h"], s["dx_in"], s["out"],
                               s["dq"], s["dp"], s["workspace"], scale=s["scale"], ranks=s["ranks"])
    return {"dx": s["out"], "dq": s["dq"], "dp": s["dp"]}


# ---- the same in 64 bits ----------------------------------------------------------------------
def _exact_adapter(s):
    """Adapter by adapter, on the rows that have it."""
    case = s["case"]
    forward = case["op"] == "forward"
    d = {k: s[k].double() for k in ("x", "q", "p", "scale") + (("y_in",) if forward else ("dy", "dx_in", "h"))}
    if forward:
        out = {"y": d["y_in"], "h": torch.zeros(case["rows"], case["r"], device=DEV, dtype=torch.float64)}
    else:
        out = {"dx": d["dx_in"], "dq": torch.zeros_like(d["q"]), "dp": torch.zeros_like(d["p"])}
    for a, rank in enumerate(_ranks(case)):
        at = (s["ids"] == a).nonzero()[:, 0]
        q, p, scale = d["q"][a, :rank], d["p"][a, :rank], d["scale"][a]
        if forward:
            h = torch.mm(d["x"][at], q.t())
            out["h"][at, :rank] = h
            out["y"][at] += scale * torch.mm(h, p)
        else:
            g = scale * torch.mm(d["dy"][at], p.t())
            out["dx"][at] += torch.mm(g, q)
            out["dq"][a, :rank] = torch.mm(g.t(), d["x"][at])
            out["dp"][a, :rank] = scale * torch.mm(d["h"][at, :rank].t(), d["dy"][at])
    return out


def _nearest(value, top, floor):
    """Groups of values as the nearest of the squares 0, 1, 4 .. top^2 of a unit that takes the largest to
    the last; with floor != 0 nothing but zero becomes zero.  Values and units."""
    value = value.view(-1, GROUP)
    unit = value.abs().amax(1, keepdim=True) / top ** 2
    root = torch.floor(torch.sqrt(value.abs() / torch.where(unit > 0, unit, 1.0)) + 0.5).clamp(max=top)
    if floor:
        root = torch.where(value != 0, root.clamp(min=floor), root)
    return (torch.sign(value) * root ** 2 * unit).view(-1), unit.view(-1)


def _exact_adamw(s):
    case, t, n = s["case"], s["step"], s["decayed"]
    p, g = s["param"].double(), s["grad"].double()
    norm = s["norm"].double()
    if norm > 1:
        g /= norm
    if case["bits"] == 8:
        m, v = (s[k].double().view(-1, GROUP) for k in "mv")
        m = (torch.sign(m) * m ** 2 * s["m_scale"].double()[:, None]).view(-1)
        v = ((v ** 2 * s["v_scale"].double()[:, None]) ** 2).view(-1)
    else:
        m, v = s["m"].double(), s["v"].double()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    p[:n] -= LR * DECAY * p[:n]
    p -= LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    out = {"param": p, **({"copy": p} if case["copy"] else {})}
    if case["bits"] == 8:
        m, out["m_scale"] = _nearest(m, 127, 0)
        root, out["v_scale"] = _nearest(torch.sqrt(v), 255, 1)
        v = root ** 2
    return dict(out, m=m, v=v)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return {"norm": torch.linalg.vector_norm(s["grad"].double())}
    return _exact_adamw(s) if case["op"] == "adamw" else _exact_adapter(s)
