"""Inner steps of K workers that share one weight matrix in HBM and differ by low-rank adapters.

Only sequencing lives here, as in the stage driver: the shared projection is a plain product, what
stands beside it and the optimizer are entry points of the HIP library.

    forward   y  = x theta_g^T                                   plain product of the working copy
              y += s_a P_a Q_a^T x  for the rows of worker a     dlcx_adapter_forward
    backward  dx = dy theta_g,  dx += ...,  dP_a, dQ_a           plain product, dlcx_adapter_backward
    update    norm of each worker's gradients, AdamW             dlcx_grad_norm, dlcx_adamw
    outer     delta_a = e_a - s_a P_a Q_a^T                      dlcx_decompress
              and on as in Alg. 2: the replicas theta_l,a = theta_g + s_a P_a Q_a^T are never formed

With the shared weights in 8 bits the plain products become dlcx_fp8_quantize and dlcx_fp8_product, a norm in front of
them (dlcx_rms_norm) writes its output in both forms, and the adapters may read their rows with dropout (dlcx_dropout),
whose mask is drawn again in the backward pass.

`python -m paper_2506_21263_amd.inner` trains two workers beside a 512 x 512 matrix towards a synthetic
teacher, outer step after outer step, and prints the losses.
"""
import argparse
import itertools
import math

import torch

from . import (BF16, F32, MMA_FMA, PHASE_P, PHASE_Q, STATE_GROUP, adapter_desc, desc, dlcx_adamw,
               dlcx_adapter_backward, dlcx_adapter_forward, dlcx_adapter_route,
               dlcx_adapter_route_bytes, dlcx_adapter_workspace_bytes, dlcx_compress_average,
               dlcx_decompress, dlcx_dropout, dlcx_fp8_product, dlcx_fp8_product_workspace_bytes, dlcx_fp8_quantize,
               dlcx_grad_norm, dlcx_orthonormalize, dlcx_outer_nesterov, dlcx_rms_norm, dlcx_rms_norm_backward,
               dlcx_rms_norm_workspace_bytes, dlcx_tensor_table, dlcx_tensor_table_bytes, dlcx_workspace_bytes,
               fp8_empty, tensor)


def _as_stream(stream):
    """The stream of a call's `stream` argument: None (the current one), a handle or a stream."""
    if stream is None:
        return torch.cuda.current_stream()
    return torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream


class Order:
    """Buffers that are written on one stream and used on another: the other waits, and the memory is not given to
    anybody else before it is through.  A graph is captured after whatever it uses is there."""

    def __init__(self, stream=None):
        self.stream = _as_stream(stream)

    def enter(self, stream, buffers):
        """The stream of a call that uses the buffers."""
        stream = _as_stream(stream)
        if stream != self.stream:
            with torch.cuda.stream(stream):
                if torch.cuda.is_current_stream_capturing():
                    return stream
            stream.wait_stream(self.stream)
            for x in buffers:
                x.record_stream(stream)
            self.stream = stream
        return stream


class Route:
    """Which rows of a batch belong to which adapter; one route serves every projection of the batch.  With a stream
    it is formed there (where `ids` has to be), and the calls that take it wait for it."""

    def __init__(self, ids, count, stream=None):
        self.ids, self.order = ids, Order(stream)
        with torch.cuda.stream(self.order.stream):
            self.table = torch.empty(dlcx_adapter_route_bytes(ids.numel(), count), device=ids.device,
                                     dtype=torch.uint8)
            dlcx_adapter_route(ids, count, self.table)


class AdamW:
    """AdamW over a list of parameters with given gradient buffers: moments of 32 or 8 bits, clipping
    by the gradients' own norm (max_norm > 0), bf16 copies of fp32 parameters where wanted.
    decays[i] is the weight decay of parameter i.  Moments of 8 bits (nearest codes) do not follow gradients of a
    group of 128 that fade unevenly at betas[1] above 0.992: that wants bits=32.

    With clipping, a step whose norm is not finite leaves everything as it was, and does not count: `step` looks at
    the norm of the step before, which the GPU has long formed by then, `taken` at the last one's.  (Steps that
    are captured into a graph are counted as they are captured.)"""

    def __init__(self, params, grads, lr, betas=(0.9, 0.95), eps=1e-8, decays=None, copies=None,
                 bits=32, max_norm=0.0):
        self.lr, self.betas, self.eps, self.max_norm, self.t = lr, betas, eps, max_norm, 0
        dev = params[0].device
        self.norm = torch.zeros(1, device=dev)
        self.norm_host = torch.empty(1, pin_memory=True)
        self.norm_there = None  # event: norm_host holds the norm of the last step
        self.moments = []
        tensors = []
        for i, p in enumerate(params):
            if bits == 8:
                groups = -(-p.numel() // STATE_GROUP)
                state = dict(m=torch.zeros(p.shape, device=dev, dtype=torch.int8),
                             v=torch.zeros(p.shape, device=dev, dtype=torch.uint8),
                             m_scale=torch.zeros(groups, device=dev),
                             v_scale=torch.zeros(groups, device=dev))
            else:
                state = dict(m=torch.zeros(p.shape, device=dev), v=torch.zeros(p.shape, device=dev))
            self.moments.append(state)
            tensors.append(tensor(grads[i], p, copy=copies[i] if copies else None,
                                  weight_decay=decays[i] if decays else 0.0, **state))
        memory = torch.empty(dlcx_tensor_table_bytes(len(tensors)), device=dev, dtype=torch.uint8)
        self.table = dlcx_tensor_table(tensors, memory)
        self.order = Order()
        self.own = [memory, self.norm] + [x for state in self.moments for x in state.values()]

    def reset(self):
        """Moments and step count of a new run."""
        self.order.enter(None, self.own)
        self.t, self.norm_there = 0, None
        for state in self.moments:
            for x in state.values():
                x.zero_()

    def taken(self):
        """Steps that changed something."""
        if self.norm_there is not None:
            self.norm_there.synchronize()
            self.norm_there = None
            self.t -= not math.isfinite(float(self.norm_host))
        return self.t

    def step(self, stream=None):
        """One step, on `stream` (gradients and parameters have to be there) after whatever came before."""
        clip = self.max_norm > 0
        with torch.cuda.stream(self.order.enter(stream, self.own)):
            capturing = torch.cuda.is_current_stream_capturing()  # where no event is waited for
            self.t = (self.t if capturing else self.taken()) + 1
            if clip:
                dlcx_grad_norm(self.table, self.norm)
            dlcx_adamw(self.table, self.lr, self.betas[0], self.betas[1], self.eps, self.t,
                       norm=self.norm if clip else None, max_norm=self.max_norm)
            if clip and not capturing:
                self.norm_host.copy_(self.norm, non_blocking=True)
                self.norm_there = torch.cuda.Event()
                self.norm_there.record()


class Norm:
    """Root-mean-square norm in front of projections, with the addition of a residual.  What the backward pass needs
    is returned by the forward pass; the weights' gradient is left in dw."""

    def __init__(self, n, dtype=torch.bfloat16, eps=1e-5, device="cuda"):
        self.n, self.eps = n, eps
        self.weight = torch.ones(n, device=device, dtype=dtype)
        self.dw = torch.zeros(n, device=device)

    def forward(self, x, residual=None, eight=False):
        """The normalised rows, the same in 8 bits (eight; else None), and (sum, rstd) for the backward pass."""
        y = torch.empty_like(x)
        y8 = fp8_empty(x.shape[0], self.n, x.device) if eight else None
        total = torch.empty_like(x) if residual is not None else None
        rstd = torch.empty(x.shape[0], device=x.device)
        dlcx_rms_norm(x, self.weight, self.eps, residual=residual, sum_out=total, y_out=y, y8_out=y8, rstd_out=rstd)
        return y, y8, (x if residual is None else total, rstd)

    def backward(self, saved, dy, dx_in=None):
        """dx (of x and of the residual); dx_in: the gradient of the sum itself."""
        x, rstd = saved
        dx = torch.empty_like(x)
        workspace = torch.empty(dlcx_rms_norm_workspace_bytes(*x.shape), device=x.device, dtype=torch.uint8)
        dlcx_rms_norm_backward(x, self.weight, rstd, dy, dx_in, dx, self.dw, workspace)
        return dx


class AdapterProjection:
    """One projection y = x theta^T with an adapter per worker.  q0: count x r x n draws; P starts at zero,
    so a new adapter changes nothing.  Masters are fp32; the products read copies in `dtype`.

    base_bits=8 keeps theta_g in 8 bits (twice: its transpose is the backward pass's), with a scale for 128 x 128 elements;
    the rows it is multiplied by are brought to 8 bits, too.  dropout: of the rows that the adapters read in training; the
    mask hangs on `seed` and the number `draw`, another one for every step, that both passes of a step are given: an int,
    or for a step that is captured into a graph an int64 tensor of one element on the device, which the program counts up.
    Without a seed, projections with dropout are numbered as a process makes them, so that no two of them have the same
    masks; pass one where processes are to differ, or where masks are not to hang on what was made before.
    Evaluation and serving pass training=False and read the rows as they are.

    An optimizer's tensors begin at 16 bytes, so where r x m or r x n elements are not whole 16 bytes, the factors are
    stored with up to seven more columns, which `ranks` leaves out of every product: p, q, dp and dq are the first r,
    h has the stored ones."""

    _seeds = itertools.count()

    def __init__(self, theta_g, q0, scale, max_rows, dtype=torch.bfloat16, base_bits=16, dropout=0.0, seed=None):
        if base_bits not in (8, 16) or not 0.0 <= dropout < 1.0:
            raise ValueError("base_bits: 8 or 16 (the adapters' own type); dropout: from 0 up to 1")
        self.m, self.n = theta_g.shape
        self.count, self.r = q0.shape[:2]
        dev = theta_g.device
        low = dtype == torch.bfloat16
        whole = 8 if low else 4  # elements of 16 bytes
        stored = self.r
        while self.count > 1 and (stored * self.m % whole or stored * self.n % whole):
            stored += 1
        self.d = adapter_desc(self.m, self.n, stored, self.count, BF16 if low else F32)
        self.ranks = None if stored == self.r else torch.full((self.count,), self.r, device=dev, dtype=torch.int32)
        self.dtype, self.q0 = dtype, q0
        self.dropout, self.seed = dropout, seed
        if seed is None:
            self.seed = next(AdapterProjection._seeds) if dropout else 0
        self.base = self.base8 = self.base8_t = None
        if base_bits == 8:
            self.base8, self.base8_t = fp8_empty(self.m, self.n, dev), fp8_empty(self.n, self.m, dev)
            dlcx_fp8_quantize(theta_g, self.base8, self.base8_t, square=True)
        else:
            self.base = theta_g.to(dtype)
        zeros = lambda k, dt=torch.float32: torch.zeros(self.count, stored, k, device=dev, dtype=dt)  # noqa: E731
        self.stored = {name: zeros(k) for name, k in (("q", self.n), ("p", self.m), ("dq", self.n), ("dp", self.m))}
        for name, k in (("q", self.n), ("p", self.m)):
            self.stored[name + "_copy"] = zeros(k, dtype) if low else self.stored[name]
        self.q, self.p, self.dq, self.dp, self.q_copy, self.p_copy = (
            self.stored[name][:, :self.r] for name in ("q", "p", "dq", "dp", "q_copy", "p_copy"))
        self.q.copy_(q0)
        if low:
            self.q_copy.copy_(q0)
        self.scale_value = scale
        self.scale = torch.full((self.count,), scale, device=dev)
        self.workspace = torch.empty(dlcx_adapter_workspace_bytes(self.d, max_rows), device=dev,
                                     dtype=torch.uint8)

    def parameters(self, a):
        """Parameters, gradients and copies of adapter a."""
        copies = [self.p_copy[a], self.q_copy[a]] if self.dtype == torch.bfloat16 else None
        return [self.p[a], self.q[a]], [self.dp[a], self.dq[a]], copies

    def _product(self, x, w, x8=None):
        """x w^T with w in 8 bits."""
        if x8 is None:
            x8 = fp8_empty(*x.shape, x.device)
            dlcx_fp8_quantize(x, x8)
        y = torch.empty(x.shape[0], w.rows, device=x.device, dtype=x.dtype)
        workspace = torch.empty(dlcx_fp8_product_workspace_bytes(x.shape[0], w.rows, w.cols), device=x.device,
                                dtype=torch.uint8)
        dlcx_fp8_product(x8, w, None, y, workspace)
        return y

    def _drops(self, draw, training):
        """Whether the adapters read their rows with dropout."""
        if not (self.dropout and training):
            return False
        if draw is None:
            raise ValueError("draw: dropout wants a number of the step in training, the same in both passes; or training=False")
        return True

    def _drop(self, x, y_in, y_out, draw):
        number, more = (0, draw) if isinstance(draw, torch.Tensor) else (draw, None)
        dlcx_dropout(x, y_in, y_out, self.dropout, self.seed, number, more)

    def _dropped(self, x, draw, drops):
        """The rows that the adapters read."""
        if not drops:
            return x
        out = torch.empty_like(x)
        self._drop(x, None, out, draw)
        return out

    def forward(self, x, route, x8=None, draw=None, training=True):
        """x8: x in 8 bits, where a norm has written it already."""
        drops = self._drops(draw, training)
        y = x @ self.base.t() if self.base is not None else self._product(x, self.base8, x8)
        route.order.enter(None, [route.table])
        h = torch.empty(x.shape[0], self.d.r, device=x.device)
        dlcx_adapter_forward(self.d, self._dropped(x, draw, drops), route.ids, self.stored["q_copy"],
                             self.stored["p_copy"], y, y, h, self.workspace, scale=self.scale, ranks=self.ranks, route=route.table)
        return y, h

    def backward(self, x, h, dy, route, draw=None, training=True):
        """dx; the gradients of the factors are left in dq and dp."""
        drops = self._drops(draw, training)
        dx = dy @ self.base if self.base is not None else self._product(dy, self.base8_t)
        route.order.enter(None, [route.table])
        # what comes through the adapters, or the whole (with dropout it is rounded to the rows' type before it is masked and
        # added: half a step of the adapters' part, where the sum's own rounding is half a step of the whole)
        own = torch.empty_like(dx) if drops else dx
        dlcx_adapter_backward(self.d, self._dropped(x, draw, drops), dy, route.ids, self.stored["q_copy"],
                              self.stored["p_copy"], h, None if drops else dx, own, self.stored["dq"], self.stored["dp"],
                              self.workspace, scale=self.scale, ranks=self.ranks, route=route.table)
        if drops:
            self._drop(own, dx, dx, draw)
        return dx

    def fold_workspace_bytes(self, group, mma):
        """Scratch of `fold`: it packs both factors of an adapter, whatever rank the outer step compresses to."""
        return 0 if mma == MMA_FMA else dlcx_workspace_bytes(desc(self.m, self.n, self.r, 8, group, mma), 1)

    def fold(self, ef, workspace, group, mma):
        """ef[a] <- ef[a] - s P_a Q_a^T for every worker: with e_a in ef[a], its pseudo-gradient."""
        need = self.fold_workspace_bytes(group, mma)
        if need and (workspace is None or workspace.numel() < need):
            raise ValueError("workspace: %d bytes are wanted" % need)
        d = desc(self.m, self.n, self.r, 8, group, mma)
        for a in range(self.count):
            dlcx_decompress(d, self.p[a] * self.scale_value, self.q[a], None, [ef[a]],
                            workspace=workspace)

    def restart(self, theta_g):
        """The adapters of the next inner phase, beside the updated weights."""
        if self.base is not None:
            self.base.copy_(theta_g)
        else:
            dlcx_fp8_quantize(theta_g, self.base8, self.base8_t, square=True)
        self.q.copy_(self.q0)
        self.p.zero_()
        if self.dtype == torch.bfloat16:
            self.q_copy.copy_(self.q)
            self.p_copy.zero_()


class AdapterOuterStep:
    """The outer step of Alg. 2 for a projection whose workers trained adapters.  M: the matrix's outer
    state (stage.MatrixState); delayed, as in the paper: what is applied at step t is the average of
    step t - 1."""

    def __init__(self, M, lr, mu):
        self.M, self.lr, self.mu, self.t = M, lr, mu, 0
        dev = M.theta_g.device
        self.delta_hat = torch.empty_like(M.theta_g)
        self.workspace = torch.empty(max(M.workspace_bytes, dlcx_workspace_bytes(M.desc(), 1)),
                                     device=dev, dtype=torch.uint8)

    def step(self, proj):
        M = self.M
        need = proj.fold_workspace_bytes(M.group, M.mma)
        if self.workspace.numel() < need:  # adapters of a higher rank than the outer step's
            self.workspace = torch.empty(need, device=self.workspace.device, dtype=torch.uint8)
        ws = self.workspace
        self.t += 1
        if self.t >= 2:
            dlcx_decompress(M.desc(M.r_prev), M.p_hat, M.q_bar, self.delta_hat, M.ef, workspace=ws)
        proj.fold(M.ef, ws, M.group, M.mma)
        if self.t >= 2:
            dlcx_outer_nesterov(M.theta_g, M.v, self.delta_hat, self.lr, self.mu)
        d = M.desc()
        basis = M.q_bar if self.t >= 2 else M.q_in
        dlcx_compress_average(d, PHASE_P, M.ef, basis, M.codes_p, M.scales_p, M.p_hat, ws)
        dlcx_orthonormalize(M.m, M.r, M.p_hat, ws)
        dlcx_compress_average(d, PHASE_Q, M.ef, M.p_hat, M.codes_q, M.scales_q, M.q_bar, ws)
        M.r_prev = M.r
        proj.restart(M.theta_g)


def train(m=512, n=512, workers=2, r=8, rows=256, inner=20, outer=8, bits=32, dtype=torch.bfloat16,
          lr=2e-2, outer_lr=0.3, outer_mu=0.0, max_norm=1.0, seed=0, device="cuda", say=None, base_bits=16,
          dropout=0.0, norm=False):
    """Workers train adapters of rank r towards a teacher that is a rank-r step away from the shared
    weights; every `inner` steps an outer step.  base_bits, dropout: AdapterProjection's; norm: rows are normalised
    before they are projected, with weights that are the workers' common ones and stay as they are, like theta_g.  Every phase goes nearly the whole way, so with the step of
    delay an outer rate above 1/4 already overshoots a little.  Returns the losses at the phases' starts."""
    from .stage import MatrixState
    from . import MMA_F32
    gen = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device=device)  # noqa: E731
    theta = 0.02 * normal(m, n)
    teacher = theta + 0.1 * normal(m, r) @ normal(r, n) / n ** 0.5
    M = MatrixState(theta, workers, normal(2 * r, n), 8, 64, MMA_F32)
    proj = AdapterProjection(theta, normal(workers, r, n) / n ** 0.5, 1.0, workers * rows, dtype, base_bits,
                             dropout, seed)
    front = Norm(n, dtype, device=device) if norm else None
    optimizers = []
    for a in range(workers):
        params, grads, copies = proj.parameters(a)
        optimizers.append(AdamW(params, grads, lr, copies=copies, bits=bits, max_norm=max_norm))
    step = AdapterOuterStep(M, outer_lr, outer_mu)
    route = Route((torch.arange(workers * rows, device=device) // rows).to(torch.int32), workers)
    losses = []
    for t in range(outer):
        for opt in optimizers:
            opt.reset()
        for k in range(inner):
            x = normal(workers * rows, n).to(dtype)      # every worker's own batch
            x8, draw = None, t * inner + k
            if norm:
                x, x8, _ = front.forward(x, eight=base_bits == 8)
            want = x.float() @ teacher.t()
            y, h = proj.forward(x, route, x8, draw)
            off = y.float() - want
            loss = (off * off).sum(1).view(workers, rows).mean(1) / m
            proj.backward(x, h, (off * (2.0 / (rows * m))).to(dtype), route, draw)
            for opt in optimizers:
                opt.step()
            if k == 0:
                losses.append(loss.mean())
        if say:
            say("outer step %d: loss %.5f at the start, %s after %d inner steps" % (
                t + 1, float(losses[-1]), " ".join("%.5f" % v for v in loss.tolist()), inner))
        step.step(proj)
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--bits", type=int, default=32, choices=(8, 32), help="of the optimizer's moments")
    ap.add_argument("--outer", type=int, default=8)
    ap.add_argument("--inner", type=int, default=20)
    ap.add_argument("--base", type=int, default=16, choices=(8, 16), help="bits of the shared weights")
    ap.add_argument("--dropout", type=float, default=0.0, help="of the rows that the adapters read")
    ap.add_argument("--norm", action="store_true", help="rows are normalised before they are projected")
    a = ap.parse_args()
    train(bits=a.bits, outer=a.outer, inner=a.inner, base_bits=a.base, dropout=a.dropout, norm=a.norm, say=lambda s: print(s, flush=True))
