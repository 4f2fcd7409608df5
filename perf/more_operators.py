"""Performance cases of the shared projection in 8 bits: what stands before it, itself, and the dropout beside it.

K workers, or requests, share a frozen projection y = x W^T and differ by adapters.  W is kept in 8 bits:
e4m3 codes with a power of two for every 128 consecutive elements of a row, which is the largest scale's
exponent that lets the largest of them fit (code 448 at most).  A matrix of rows x cols has rows of codes
that are padded with zeros to a multiple of 128, and rows of scale bytes (exponent + 127) that are padded
to a multiple of 4.  A case is a dict of plain values whose "op" names the call:

  norm           dlcx_rms_norm: s = x + residual, y = s rstd w with rstd = 1 / sqrt(mean s^2 + eps), y rounded
                 to x's type or to 8 bits
  norm_backward  dlcx_rms_norm_backward: dx and dw of the same
  quantize       dlcx_fp8_quantize: a matrix to 8 bits along its rows; "both": its transpose along that one's
                 rows, too (a gradient is read both ways); "square": both with one scale for 128 x 128 (weights)
  product        dlcx_fp8_product: y = y_in + x w^T of two matrices in 8 bits
  dropout        dlcx_dropout: y = y_in + x mask / (1 - p), the mask from counters (Philox 4x32, ten rounds)

Results in 8 bits are returned as what they stand for (dlcx_fp8_decode), in bf16: a code has four
significant bits and a scale is a power of two, so nothing is rounded.

Sizes are those of the benchmark configurations (the matrices of an OPT-1.3B-like layer and of a ~100B dense
layer, four workers) and odd sizes around them.  All inputs are drawn on the GPU from the seed: activations
N(0, 1) whose columns differ in scale, weights N(0, 0.02^2), gradients N(0, 1e-3^2) whose rows differ.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 128                      # elements that share a scale
TOP = 448.0                      # the largest e4m3 value
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one token of one request before an OPT-1.3B projection: launches and latency count
        dict(name="norm-1-row-2048-to-8-bits", op="norm", rows=1, n=2048, dtype="bf16", residual=True, out="eight"),
        # the prompts of a dozen requests, of ragged lengths, before the dense layer's projections
        dict(name="norm-4133-rows-8192-to-8-bits", op="norm", rows=4133, n=8192, dtype="bf16", residual=True,
             out="eight"),
        # a micro-batch of each of four workers: training, with the residual's gradient
        dict(name="norm-backward-16384-rows-8192", op="norm_backward", rows=16384, n=8192, dtype="bf16",
             residual=True),
        # a short ragged batch in fp32, of an odd size that no 16-byte access fits
        dict(name="norm-backward-515-rows-2050-f32", op="norm_backward", rows=515, n=2050, dtype="f32",
             residual=False),
        # the gradient of a projection's output, for the products with the weights and with the inputs
        dict(name="quantize-16384-rows-8192-both", op="quantize", rows=16384, cols=8192, dtype="bf16", form="both"),
        # fp32 weights of an odd size, once an outer step, for forward and backward
        dict(name="quantize-2050-rows-1021-square-f32", op="quantize", rows=2050, cols=1021, dtype="f32",
             form="square"),
        # one token of one request through an OPT-1.3B projection
        dict(name="product-1-row-2048x2048", op="product", rows=1, m=2048, n=2048, out="bf16", add=False),
        # one token of each of 96 requests through the dense layer's widest projection
        dict(name="product-96-rows-28672x8192", op="product", rows=96, m=28672, n=8192, out="bf16", add=False),
        # a micro-batch of each of four workers: training and prompts
        dict(name="product-16384-rows-8192x8192", op="product", rows=16384, m=8192, n=8192, out="bf16", add=False),
        # the gradient of odd weights from 4133 rows, added to what fp32 gradients hold already
        dict(name="product-2050-rows-1021x4133-f32-added", op="product", rows=2050, m=1021, n=4133, out="f32",
             add=True),
        # what the adapters of four workers read in training, or a block's output into its residual
        dict(name="dropout-16384-rows-8192-added", op="dropout", rows=16384, cols=8192, dtype="bf16", p=0.1,
             add=True),
        # a short ragged batch in fp32
        dict(name="dropout-515-rows-2050-f32", op="dropout", rows=515, cols=2050, dtype="f32", p=0.05, add=False),
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def _side(rng, hi):
    return _log(rng, 64, hi) if rng.random() < 0.4 else 16 * _log(rng, 4, hi // 16)


def draw(rng):
    op = rng.choice(("norm", "norm", "norm_backward", "norm_backward", "quantize", "quantize", "product", "product",
                     "product", "product", "dropout", "dropout"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "product":
        rows = _log(rng, 1, 96) if rng.random() < 0.4 else _log(rng, 96, 12000)
        return dict(op=op, rows=rows, m=_side(rng, 12000), n=_side(rng, 6000), out=dtype, add=rng.random() < 0.4)
    rows, cols = _log(rng, 1, 8192), _side(rng, 8192)
    if op == "norm":
        return dict(op=op, rows=rows, n=cols, dtype=dtype, residual=rng.random() < 0.6,
                    out=rng.choice(("plain", "eight", "both")))
    if op == "norm_backward":
        return dict(op=op, rows=rows, n=cols, dtype=dtype, residual=rng.random() < 0.5)
    if op == "quantize":
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, form=rng.choice(("rows", "both", "square")))
    return dict(op=op, rows=rows, cols=cols, dtype=dtype, p=round(rng.uniform(0.01, 0.6), 3), add=rng.random() < 0.5)


# ---- what a pass cannot do without ------------------------------------------------------------
def _eight(rows, cols):
    """Bytes of a matrix in 8 bits."""
    return rows * cols + rows * -(-cols // BLOCK)


def work(case):
    op, rows = case["op"], case["rows"]
    if op == "product":
        m, n = case["m"], case["n"]
        y = rows * m * TYPES[case["out"]].itemsize * (2 if case["add"] else 1)
        return {"bytes": _eight(rows, n) + _eight(m, n) + y, "flops": 2 * rows * m * n}
    size = TYPES[case["dtype"]].itemsize
    if op == "norm":
        n = case["n"]
        each = size * ((3 if case["residual"] else 1) + (case["out"] != "eight"))
        values = 0 if case["out"] == "plain" else 2 * _eight(rows, n) + 2 * rows * n   # written, read, decoded
        return {"bytes": rows * n * each + values + rows * 4 + n * size, "flops": 5 * rows * n}
    if op == "norm_backward":
        n = case["n"]
        return {"bytes": rows * n * size * (4 if case["residual"] else 3) + rows * 4 + n * (size + 4),
                "flops": 9 * rows * n}
    cols = case["cols"]
    if op == "quantize":
        values = 2 * _eight(rows, cols) + 2 * rows * cols
        if case["form"] != "rows":
            values += 2 * _eight(cols, rows) + 2 * rows * cols
        return {"bytes": rows * cols * size + values, "flops": 3 * rows * cols}
    return {"bytes": rows * cols * size * (3 if case["add"] else 2), "flops": 2 * rows * cols}


# ---- matrices in 8 bits, in elementary operations ----------------------------------------------
def _up(x, to):
    return -(-x // to) * to


def _power(exponent):
    """2^exponent in 32 bits, exactly, from its bits in 64 (a pow or exp2 of the GPU can be a bit off)."""
    return (exponent.to(torch.int64) + 1023 << 52).view(torch.float64).float()


def _to_eight(x, square=False):
    """Codes (e4m3, rows padded with zeros) and scale bytes of a matrix's rows."""
    rows, cols = x.shape
    wide = _up(cols, BLOCK)
    v = torch.zeros(_up(rows, BLOCK) if square else rows, wide, device=DEV)
    v[:rows, :cols] = x
    largest = v.abs().view(v.shape[0], -1, BLOCK).amax(2)
    if square:
        largest = largest.view(-1, BLOCK, largest.shape[1]).amax(1).repeat_interleave(BLOCK, 0)[:rows]
        v = v[:rows]
    fraction, exponent = torch.frexp(largest)                  # largest = fraction 2^exponent, from 1/2 to 1
    exponent = exponent - 9 + (fraction > TOP / 512)
    exponent = torch.where(largest > 0, exponent.clamp(min=-127), 0)
    codes = (v.view(rows, -1, BLOCK) * _power(-exponent)[:, :, None]).view(rows, wide).to(torch.float8_e4m3fn)
    scales = torch.full((rows, _up(wide // BLOCK, 4)), 127, device=DEV, dtype=torch.uint8)
    scales[:, :wide // BLOCK] = exponent + 127
    return codes, scales


def _from_eight(codes, scales, cols):
    """What they stand for, in 32 bits."""
    rows = codes.shape[0]
    exponent = scales[:, :codes.shape[1] // BLOCK].to(torch.int32) - 127
    return (codes.float().view(rows, -1, BLOCK) * _power(exponent)[:, :, None]).view(rows, -1)[:, :cols]


# ---- inputs -----------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op, rows = case["op"], case["rows"]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device=DEV) * std

    def activations(*shape):
        return normal(*shape).mul_(normal(shape[1], std=0.7).exp_())

    def gradients(*shape):
        return normal(*shape, std=1e-3).mul_(normal(shape[0], 1, std=0.7).exp_())

    s = dict(case=case)
    if op == "product":
        m, n, dt = case["m"], case["n"], TYPES[case["out"]]
        s["x"], s["w"] = _to_eight(activations(rows, n)), _to_eight(normal(m, n, std=0.02), square=True)
        s["y_in"] = normal(rows, m).to(dt) if case["add"] else None
        s["y"] = torch.empty(rows, m, device=DEV, dtype=dt)
        if own:   # the matrices as the calls take them, and the workspace that a program keeps
            import paper_2506_21263_amd as dlcx
            s["x8"], s["w8"] = (dlcx.fp8(*s[k], n) for k in "xw")
            s["workspace"] = torch.empty(dlcx.dlcx_fp8_product_workspace_bytes(rows, m, n), device=DEV, dtype=torch.uint8)
        return s
    dt = TYPES[case["dtype"]]
    if op in ("norm", "norm_backward"):
        n = case["n"]
        s["x"], s["weight"] = activations(rows, n).to(dt), (1 + normal(n, std=0.2)).to(dt)
        if op == "norm_backward":
            s["rstd"] = (s["x"].float().square().mean(1) + EPS).rsqrt()
            s["dy"] = gradients(rows, n).to(dt)
            s["dx_in"] = gradients(rows, n).to(dt) if case["residual"] else None
            s["dx"], s["dw"] = torch.empty(rows, n, device=DEV, dtype=dt), torch.empty(n, device=DEV)
            if own:
                import paper_2506_21263_amd as dlcx
                s["workspace"] = torch.empty(dlcx.dlcx_rms_norm_workspace_bytes(rows, n), device=DEV, dtype=torch.uint8)
            return s
        s["residual"] = activations(rows, n).to(dt) if case["residual"] else None
        s["rstd"] = torch.empty(rows, device=DEV)
        s["sum"] = torch.empty(rows, n, device=DEV, dtype=dt) if case["residual"] else None
        s["y"] = torch.empty(rows, n, device=DEV, dtype=dt) if case["out"] != "eight" else None
        s["values"] = torch.empty(rows, n, device=DEV, dtype=torch.bfloat16) if case["out"] != "plain" else None
        if own:
            import paper_2506_21263_amd as dlcx
            s["y8"] = dlcx.fp8_empty(rows, n) if case["out"] != "plain" else None
        return s
    cols = case["cols"]
    if op == "quantize":
        s["x"] = (normal(rows, cols, std=0.02) if case["form"] == "square" else gradients(rows, cols)).to(dt)
        s["values"] = torch.empty(rows, cols, device=DEV, dtype=torch.bfloat16)
        s["values_t"] = None if case["form"] == "rows" else torch.empty(cols, rows, device=DEV, dtype=torch.bfloat16)
        if own:
            import paper_2506_21263_amd as dlcx
            s["x8"] = dlcx.fp8_empty(rows, cols)
            s["x8_t"] = None if case["form"] == "rows" else dlcx.fp8_empty(cols, rows)
        return s
    s["x"] = activations(rows, cols).to(dt)
    s["y_in"] = activations(rows, cols).to(dt) if case["add"] else None
    s["y"] = torch.empty(rows, cols, device=DEV, dtype=dt)
    s["seed"] = (0x9E3779B97F4A7C15 ^ seed) % 2 ** 64      # of the run
    s["offset"] = ((3 << 32) + 7 * seed) % 2 ** 64         # of the step and the place in the model
    return s


# ---- the operators ----------------------------------------------------------------------------
LOW = 0xFFFFFFFF


def _bits(groups, seed, offset):
    """Eight numbers of 16 bits for every group of eight elements (64-bit products that wrap, masked)."""
    group = torch.arange(groups, device=DEV)
    c0, c1 = group & LOW, group >> 32
    c2, c3 = torch.full_like(group, offset & LOW), torch.full_like(group, offset >> 32)
    k0, k1 = seed & LOW, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & LOW) ^ c1 ^ k0, b & LOW, (a >> 32 & LOW) ^ c3 ^ k1, a & LOW
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    words = torch.stack((c0, c1, c2, c3), 1)
    return torch.stack((words & 0xFFFF, words >> 16), 2).view(groups * 8)


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "product":
        x, w = (_from_eight(*s[k], case["n"]) for k in "xw")
        y = x @ w.t()
        return {"y": (y if s["y_in"] is None else s["y_in"].float() + y).to(s["y"].dtype)}
    if op == "quantize":
        square = case["form"] == "square"
        out = {"values": _from_eight(*_to_eight(s["x"], square), case["cols"]).to(torch.bfloat16)}
        if case["form"] != "rows":
            out["values_t"] = _from_eight(*_to_eight(s["x"].t(), square), case["rows"]).to(torch.bfloat16)
        return out
    if op == "dropout":
        x = s["x"]
        threshold = round(case["p"] * 65536)
        kept = _bits(-(-x.numel() // 8), s["seed"], s["offset"])[:x.numel()].view(x.shape) >= threshold
        y = torch.where(kept, x.float() * (65536 / (65536 - threshold)), 0.0)
        return {"y": (y if s["y_in"] is None else s["y_in"].float() + y).to(x.dtype)}
    x, w = s["x"].float(), s["weight"].float()
    if op == "norm_backward":
        rstd, dy = s["rstd"][:, None], s["dy"].float()
        hat, g = x * rstd, dy * w
        dx = rstd * (g - hat * (g * hat).mean(1, keepdim=True))
        return {"dx": (dx if s["dx_in"] is None else s["dx_in"].float() + dx).to(s["x"].dtype),
                "dw": (dy * hat).sum(0)}
    out = {}
    if s["residual"] is not None:
        out["sum"] = (x + s["residual"].float()).to(s["x"].dtype)
        x = out["sum"].float()
    out["rstd"] = (x.square().mean(1) + EPS).rsqrt()
    y = x * out["rstd"][:, None] * w
    if case["out"] != "eight":
        out["y"] = y.to(s["x"].dtype)
    if case["out"] != "plain":
        out["values"] = _from_eight(*_to_eight(y), case["n"]).to(torch.bfloat16)
    return out


def run(s):
    if not own:
        return _plain(s)
    import paper_2506_21263_amd as dlcx
    case = s["case"]
    op = case["op"]
    if op == "product":
        dlcx.dlcx_fp8_product(s["x8"], s["w8"], s["y_in"], s["y"], s["workspace"])
        return {"y": s["y"]}
    if op == "quantize":
        dlcx.dlcx_fp8_quantize(s["x"], s["x8"], s["x8_t"], square=case["form"] == "square")
        out = {}
        for name, of in (("values", "x8"), ("values_t", "x8_t")):
            if s[name] is not None:
                dlcx.dlcx_fp8_decode(s[of], s[name])
                out[name] = s[name]
        return out
    if op == "dropout":
        dlcx.dlcx_dropout(s["x"], s["y_in"], s["y"], case["p"], s["seed"], s["offset"])
        return {"y": s["y"]}
    if op == "norm_backward":
        dlcx.dlcx_rms_norm_backward(s["x"], s["weight"], s["rstd"], s["dy"], s["dx_in"], s["dx"], s["dw"],
                                    s["workspace"])
        return {"dx": s["dx"], "dw": s["dw"]}
    dlcx.dlcx_rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], sum_out=s["sum"], y_out=s["y"],
                       y8_out=s["y8"], rstd_out=s["rstd"])
    if s["values"] is not None:
        dlcx.dlcx_fp8_decode(s["y8"], s["values"])
    return {k: s[k] for k in ("sum", "rstd", "y", "values") if s[k] is not None}


# ---- the same in 64 bits ----------------------------------------------------------------------
def _nearest(x, tile):
    """The nearest e4m3 multiples of each tile's power of two (tile: rows and columns that share one)."""
    rows, cols = x.shape
    a, b = tile
    v = torch.zeros(_up(rows, a), _up(cols, b), device=DEV, dtype=torch.float64)
    v[:rows, :cols] = x
    v = v.view(v.shape[0] // a, a, -1, b)
    top = v.abs().amax((1, 3), keepdim=True)
    unit = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, TOP) / TOP)).clamp(min=-127))
    v = v / unit
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step * unit).reshape(_up(rows, a), -1)[:rows, :cols]


def _of_bytes(codes, scales, cols):
    """Sign, exponent and fraction of the codes, times the scales."""
    byte = codes.view(torch.uint8)[:, :cols].to(torch.int64)
    e, f = (byte >> 3) & 15, (byte & 7).double()
    value = torch.where(e > 0, (8 + f) * torch.exp2(e.double() - 10), f * 2.0 ** -9)
    unit = torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, 1)[:, :cols]
    return torch.where(byte > 127, -value, value) * unit


def _times(a, b):
    """High and low 32 bits of products of 32-bit numbers, b one number: no step passes 2^49."""
    b0, b1 = b & 0xFFFF, b >> 16
    low, high = a * b0, a * b1
    middle = (low >> 16) + (high & 0xFFFF)
    return (high >> 16) + (middle >> 16), ((middle & 0xFFFF) << 16) | (low & 0xFFFF)


def _exact_kept(case, seed, offset):
    rows, cols = case["rows"], case["cols"]
    at = torch.arange(-(-rows * cols // 8), device=DEV)
    c = [at % 2 ** 32, at // 2 ** 32, torch.zeros_like(at) + offset % 2 ** 32, torch.zeros_like(at) + offset // 2 ** 32]
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for turn in range(10):
        (h0, l0), (h2, l2) = _times(c[0], 0xD2511F53), _times(c[2], 0xCD9E8D57)
        c = [h2 ^ c[1] ^ ((key[0] + turn * 0x9E3779B9) % 2 ** 32), l2, h0 ^ c[3] ^ ((key[1] + turn * 0xBB67AE85) % 2 ** 32), l0]
    kept = torch.empty(at.numel(), 8, device=DEV, dtype=torch.bool)
    for j in range(8):
        kept[:, j] = (c[j // 2] // (65536 if j % 2 else 1)) % 65536 >= round(case["p"] * 65536)
    return kept.view(-1)[:rows * cols].view(rows, cols)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "product":
        y = torch.mm(_of_bytes(*s["x"], case["n"]), _of_bytes(*s["w"], case["n"]).t())
        return {"y": y if s["y_in"] is None else y + s["y_in"].double()}
    x = s["x"].double()
    if op == "quantize":
        tile = (BLOCK, BLOCK) if case["form"] == "square" else (1, BLOCK)
        out = {"values": _nearest(x, tile)}
        if case["form"] != "rows":
            out["values_t"] = _nearest(x.t(), tile)
        return out
    if op == "dropout":
        keep = 1 - round(case["p"] * 65536) / 65536
        y = x * _exact_kept(case, s["seed"], s["offset"]) / keep
        return {"y": y if s["y_in"] is None else y + s["y_in"].double()}
    w, n = s["weight"].double(), case["n"]
    if op == "norm_backward":
        dy, rstd = s["dy"].double(), s["rstd"].double()[:, None]
        dw = torch.einsum("ti,ti->i", dy, x * rstd)
        along = ((dy * w * x).sum(1, keepdim=True) * rstd ** 3 / n)
        dx = dy * w * rstd - x * along
        return {"dx": dx if s["dx_in"] is None else dx + s["dx_in"].double(), "dw": dw}
    out = {}
    if s["residual"] is not None:
        out["sum"] = x + s["residual"].double()
        x = out["sum"].to(s["x"].dtype).double()       # what is stored is what is normalised
    out["rstd"] = 1 / torch.sqrt((x * x).sum(1) / n + EPS)
    y = x * out["rstd"][:, None] * w
    if case["out"] != "eight":
        out["y"] = y
    if case["out"] != "plain":
        out["values"] = _nearest(y, (1, BLOCK))
    return out
