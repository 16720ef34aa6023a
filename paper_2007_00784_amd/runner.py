"""Drives a whole synthetic workload (a layer set) through the C-ABI library.

Holds device buffers and call order only: every arithmetic step is a library call.  Used by the
benchmark and by the full-size parity tests.

Everything a runner does goes to the stream that was the current one when it was made; inputs from another stream and
results used on one are the caller's to order.
"""
import contextlib

import numpy as np
import torch

from . import kfac as K
from . import synthetic as S


@contextlib.contextmanager
def own_stream(run, *inputs):
    """torch's operations between the library's calls of a runner go where those do, whatever the caller's stream is, and behind what that stream holds by now
    (a mask that was just made, say)."""
    now = torch.cuda.current_stream(run.dev)
    if now == run.stream:
        yield
        return
    run.stream.wait_stream(now)
    for t in inputs:
        if t.is_cuda:
            t.record_stream(run.stream)
    with torch.cuda.stream(run.stream):
        yield


class KfacRunner:
    def __init__(self, wl, device="cuda:0", n_updates=2, batch=None, layers=None, verbose=False):
        self.wl = wl
        self.dev = torch.device(device)
        self.N = wl.batch if batch is None else batch
        self.layer_ids = list(range(len(wl.layers))) if layers is None else list(layers)
        self.layers = [wl.layers[i] for i in self.layer_ids]
        self.n_updates = n_updates
        self.dt = torch.bfloat16 if wl.bf16 else torch.float32
        self.x, self.g = [], []          # [update][layer] device tensors
        self.gradw_master = []
        for u in range(n_updates):
            xs, gs = [], []
            for li in self.layer_ids:
                t = S.layer_inputs(wl, li, update=u, batch=self.N, want=("x", "g"))
                xs.append(self._up(t["x"]))
                gs.append(self._up(t["g"]))
                if verbose:
                    print("generated update %d layer %d" % (u, li), flush=True)
            self.x.append(xs)
            self.g.append(gs)
        # all gradients live in one flat buffer (and so do their masters), so that restoring them before an
        # in-place preconditioning is a single device copy
        gw = [S.layer_inputs(wl, li, batch=self.N, want=("gradw",))["gradw"] for li in self.layer_ids]
        offs = np.cumsum([0] + [(g.size + 63) // 64 * 64 for g in gw])
        self.gradw_master_flat = torch.zeros(int(offs[-1]), dtype=self.dt, device=self.dev)
        self.grad_flat = torch.zeros_like(self.gradw_master_flat)
        for j, g in enumerate(gw):
            view = self.gradw_master_flat[int(offs[j]):int(offs[j]) + g.size].view(g.shape)
            view.copy_(self._up(g))
            self.gradw_master.append(view)
        f32 = dict(dtype=torch.float32, device=self.dev)
        self.A = [torch.zeros((l.d_a, l.d_a), **f32) for l in self.layers]
        self.G = [torch.zeros((l.d_g, l.d_g), **f32) for l in self.layers]
        self.QA = [torch.zeros_like(a) for a in self.A]
        self.QG = [torch.zeros_like(g) for g in self.G]
        self.lamA = [torch.zeros(l.d_a, **f32) for l in self.layers]
        self.lamG = [torch.zeros(l.d_g, **f32) for l in self.layers]
        self.grad = [self.grad_flat[int(offs[j]):int(offs[j]) + g.size].view(g.shape) for j, g in enumerate(gw)]
        # every unfolded layer keeps its own patch slab, so all factor updates go out as one batch
        self.patches = [torch.empty((l.d_a - 1) * l.T * self.N, dtype=self.dt, device=self.dev) if l.needs_unfold else None
                        for l in self.layers]
        dims = [l.d_a for l in self.layers] + [l.d_g for l in self.layers]
        need = K.kfac_eig_workspace_bytes(dims)
        need = max(need, K.kfac_update_factors_workspace_bytes(self._factor_items(0, 0.0, sizing=True)))
        need = max(need, K.kfac_precondition_workspace_bytes([(l.d_a, l.d_g) for l in self.layers]))
        need = max(need, K.kfac_grad_norm_workspace_bytes(K.grad_items(self.grad)))
        need = max(need, K.kfac_workspace_bytes(max(dims), 1, max(l.rows(self.N) for l in self.layers)))  # SYRK partials, precondition
        self.ws = torch.empty(need + 4096, dtype=torch.uint8, device=self.dev)
        self.stream = torch.cuda.current_stream(self.dev)
        self.ctx = K.kfac_create(self.dev.index or 0, self.stream.cuda_stream, self.ws)
        self.norm, self.coef = torch.zeros(1, **f32), torch.zeros(1, **f32)
        self.eig_info = None
        self._marshalled = {}    # item arrays of the batched calls, marshalled once per distinct argument set

    def _up(self, a):
        t = torch.from_numpy(np.ascontiguousarray(a)).to(self.dev)
        return t.to(torch.bfloat16) if self.wl.bf16 else t

    def close(self):
        torch.cuda.synchronize()
        if self.ctx is not None:
            K.kfac_destroy(self.ctx)
            self.ctx = None

    # ---- phases ----
    def _factor_items(self, upd, decay, sizing=False):
        N = self.N
        code = K.KFAC_BF16 if self.wl.bf16 else K.KFAC_F32
        items = []
        for i, l in enumerate(self.layers):
            R = N * l.T
            lay = K.KFAC_LAYOUT_RD if l.fc else K.KFAC_LAYOUT_NDT
            T = 1 if l.fc else l.T
            if sizing:
                src = g = FA = FG = None
            else:
                src = self.patches[i] if l.needs_unfold else self.x[upd][i]   # [N][C][H*W] is already the patch slab
                g, FA, FG = self.g[upd][i], self.A[i], self.G[i]
            items.append(dict(X=src, dtype=code, layout=lay, N=N, d=l.d_a - 1, T=T, append_ones=1, scale=1.0 / R,
                              decay=decay, F=FA))
            items.append(dict(X=g, dtype=code, layout=lay, N=N, d=l.d_g, T=T, append_ones=0, scale=1.0 / R,
                              decay=decay, F=FG))
        return items

    def update_factors(self, upd, decay, batched=True):
        idx = [i for i, l in enumerate(self.layers) if l.needs_unfold]
        if batched and idx:
            K.kfac_unfold_batched(self.ctx, [self.x[upd][i] for i in idx],
                                  [(self.layers[i].k, self.layers[i].k, self.layers[i].stride, self.layers[i].pad) for i in idx],
                                  [self.patches[i] for i in idx])
        else:
            for i in idx:
                l = self.layers[i]
                K.kfac_unfold(self.ctx, self.x[upd][i], l.k, l.k, l.stride, l.pad, self.patches[i])
        if batched:
            key = ("factors", upd, float(decay))
            if key not in self._marshalled:
                self._marshalled[key] = K.factor_items(self._factor_items(upd, decay))
            K.kfac_update_factors_batched(self.ctx, self._marshalled[key])
            return
        for it in self._factor_items(upd, decay):
            K.kfac_update_factors(self.ctx, it["X"], it["layout"], it["N"], it["d"], it["T"], it["append_ones"],
                                  it["scale"], it["decay"], it["F"], dtype=it["dtype"])

    def eig(self, **kw):
        self.eig_info = K.kfac_eig(self.ctx, self.A + self.G, self.QA + self.QG, self.lamA + self.lamG, **kw)
        return self.eig_info

    def restore_gradients(self):
        """Fresh gradients for the next in-place preconditioning (one device copy of the flat master buffer): what
        the backward pass of a training iteration delivers."""
        with own_stream(self):
            self.grad_flat.copy_(self.gradw_master_flat)

    def precondition(self, damping=None, kappa=None, lr=None, split_f16=None, restore=True):
        """In-place preconditioning of the gradients (restored from their masters first unless restore=False); with
        kappa and lr also the gradient scaling nu (left in self.nu, a device tensor).  split_f16 defaults to the
        workload's gradient type: bf16 gradients (rounding 4e-3) go through the split-fp16 GEMM chain (error 1e-6),
        fp32 ones through fp32."""
        gamma = self.wl.damping if damping is None else damping
        split = self.wl.bf16 if split_f16 is None else split_f16
        if restore:
            self.restore_gradients()
        key = ("precond", float(gamma), bool(split))
        if key not in self._marshalled:
            self._marshalled[key] = K.precond_items(self.QA, self.lamA, self.QG, self.lamG, gamma, self.grad, split_f16=split)
        if kappa is None:
            K.kfac_precondition_batched(self.ctx, items=self._marshalled[key])
        else:
            with own_stream(self):
                self.nu = torch.zeros(1, dtype=torch.float32, device=self.dev)
            K.kfac_precondition_batched_scaled(self.ctx, kappa=kappa, lr=lr, nu=self.nu, items=self._marshalled[key])

    def clip(self, max_norm):
        """The gradients, in place, times min(1, max_norm / their global norm).  The norm and what they were multiplied with stay on the GPU: self.norm
        and self.coef."""
        if "clip" not in self._marshalled:
            self._marshalled["clip"] = K.grad_items(self.grad, self.grad)
        K.kfac_clip_grads_batched(self.ctx, self._marshalled["clip"], max_norm, self.norm, self.coef)

    # ---- the explicit-inverse method (Sec. II-C, Eq. (kfac-damped)): the paper's other way to the same step ----
    def invert_factors(self, damping=None):
        """(A + gamma I)^-1 and (G + gamma I)^-1 of every layer by blocked Cholesky (buffers allocated on first use)."""
        gamma = self.wl.damping if damping is None else damping
        if not hasattr(self, "Ainv"):
            with own_stream(self):
                self.Ainv = [torch.empty_like(a) for a in self.A]
                self.Ginv = [torch.empty_like(g) for g in self.G]
        K.kfac_invert_factors(self.ctx, self.A + self.G, gamma, self.Ainv + self.Ginv)

    def precondition_inverse(self, restore=True):
        """grad <- Ginv grad Ainv for every layer, in place."""
        if restore:
            self.restore_gradients()
        if "precond_inv" not in self._marshalled:
            self._marshalled["precond_inv"] = K.precond_inv_items(self.Ainv, self.Ginv, self.grad)
        K.kfac_precondition_inverse_batched(self.ctx, items=self._marshalled["precond_inv"])

    # ---- algorithmic work of one step (flops, bytes) ----
    def work(self):
        N = self.N
        esz = 2 if self.wl.bf16 else 4
        w = dict(syrk_flops=0.0, precond_flops=0.0, unfold_bytes=0.0, ema_bytes=0.0, sum_d3=0.0)
        for l in self.layers:
            R = N * l.T
            w["syrk_flops"] += R * (l.d_a * (l.d_a + 1.0) + l.d_g * (l.d_g + 1.0))
            w["precond_flops"] += 4.0 * l.d_a * l.d_g * (l.d_a + l.d_g)
            if l.needs_unfold:
                w["unfold_bytes"] += esz * (N * l.c_in * l.h_in * l.h_in + R * (l.d_a - 1.0))
            w["ema_bytes"] += 8.0 * (l.d_a ** 2 + l.d_g ** 2)
            w["sum_d3"] += float(l.d_a) ** 3 + float(l.d_g) ** 3
        return w


def device_of(device):
    """A device with its number: "cuda" is the current one, for the tensors as for the library's context."""
    d = torch.device(device)
    return torch.device(d.type, torch.cuda.current_device()) if d.type == "cuda" and d.index is None else d


class ExpertRunner:
    """A layer of experts through a training step with the preconditioner: products, both gradients, every expert's factors, their
    eigendecompositions, the preconditioned gradient and the optimizer step that writes the weights which the next products read.

    The rows of x and g are sorted by expert, offsets (int32 [experts + 1], on the GPU) say where each one's begin.  Parameters are kept in fp32 with their
    bias as last column; bf16 layers multiply with a bf16 copy of them that the optimizer step writes.  seed: of the rounding of an 8-bit state.
    more_workspace: bytes that the context's workspace has at least, for calls besides this layer's.
    """
    # At step t a gradient as large as the average moves sqrt(v) by 1 / (2 t) (beta2 near 1), which up to the eighth is half the distance of two
    # codes at least: until then an 8-bit state is rounded to nearest, which is off by less; from then on by the seed, or it would stand still.
    NEAREST_STEPS = 8

    def __init__(self, experts, rows, d_in, d_out, bias=True, bf16=True, state_bits=32, damping=1e-3, device="cuda:0", seed=1, more_workspace=0):
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.dev = device_of(device)
        self.experts, self.rows, self.d_in, self.d_out, self.bias, self.damping = experts, rows, d_in, d_out, bool(bias), damping
        self.dt = torch.bfloat16 if bf16 else torch.float32
        dA = d_in + int(self.bias)
        f32 = dict(dtype=torch.float32, device=self.dev)
        self.param = torch.zeros((experts, d_out, dA), **f32)
        self.weight = torch.zeros_like(self.param, dtype=self.dt) if bf16 else self.param
        self.grad = torch.zeros_like(self.param)
        self.y = torch.zeros((rows, d_out), dtype=self.dt, device=self.dev)
        self.dx = torch.zeros((rows, d_in), dtype=self.dt, device=self.dev)
        self.A, self.G = torch.zeros((experts, dA, dA), **f32), torch.zeros((experts, d_out, d_out), **f32)
        self.QA, self.QG = torch.zeros_like(self.A), torch.zeros_like(self.G)
        self.lamA, self.lamG = torch.zeros((experts, dA), **f32), torch.zeros((experts, d_out), **f32)
        self.state_bits = state_bits
        self.state = self._state(self.param)
        self._grads = K.grad_items([self.grad])
        self.norm, self.coef = torch.zeros(1, **f32), torch.zeros(1, **f32)
        self.steps, self.seed = 0, seed
        dims = [dA] * experts + [d_out] * experts
        need = max(K.kfac_eig_workspace_bytes(dims), K.kfac_precondition_workspace_bytes([(dA, d_out)] * experts),
                   K.kfac_experts_workspace_bytes(experts, rows, d_in, d_out, self.bias, K.KFAC_BF16 if bf16 else K.KFAC_F32),
                   K.kfac_grad_norm_workspace_bytes(self._grads), more_workspace)
        self.ws = torch.empty(need + 4096, dtype=torch.uint8, device=self.dev)
        self.stream = torch.cuda.current_stream(self.dev)
        self.ctx = K.kfac_create(self.dev.index, self.stream.cuda_stream, self.ws)
        self._adamw = K.adamw_items([self._item(self.param, self.grad, self.state, self.weight)])
        self._precond = K.precond_items(list(self.QA), list(self.lamA), list(self.QG), list(self.lamG), damping, list(self.grad))

    def _state(self, param):
        n = param.numel()
        if self.state_bits == 32:
            return {k: torch.zeros(n, dtype=torch.float32, device=self.dev) for k in ("m", "v")}
        state = {k: torch.zeros(n, dtype=torch.uint8, device=self.dev) for k in ("m", "v")}
        state.update({k: torch.zeros((n + 127) // 128, dtype=torch.uint8, device=self.dev) for k in ("m_scale", "v_scale")})
        return state

    def _item(self, param, grad, state, weight):
        return dict(param=param, grad=grad, **state, **(dict(copy=weight) if weight is not param else {}))

    def close(self):
        torch.cuda.synchronize(self.dev)
        if self.ctx is not None:
            K.kfac_destroy(self.ctx)
            self.ctx = None

    def load(self, param):
        """The parameters [experts, d_out, d_in + bias], and the weights that the products read."""
        with own_stream(self, param):
            self.param.copy_(param)
            if self.weight is not self.param:
                self.weight.copy_(self.param)

    def forward(self, x, offsets):
        K.kfac_experts_forward(self.ctx, x, self.weight, offsets, self.y, append_ones=self.bias)
        return self.y

    def backward(self, x, g, offsets, accumulate=False):
        """The input's gradient (returned) and every expert's (self.grad) from the output's."""
        K.kfac_experts_input_grad(self.ctx, g, self.weight, offsets, self.dx, append_ones=self.bias)
        K.kfac_experts_weight_grad(self.ctx, g, x, offsets, self.grad, append_ones=self.bias, accumulate=accumulate)
        return self.dx

    def update_factors(self, x, g, offsets, decay):
        K.kfac_update_factors_experts(self.ctx, x, offsets, self.A, append_ones=self.bias, decay=decay)
        K.kfac_update_factors_experts(self.ctx, g, offsets, self.G, decay=decay)

    def eig(self, **kw):
        return K.kfac_eig(self.ctx, list(self.A) + list(self.G), list(self.QA) + list(self.QG), list(self.lamA) + list(self.lamG), **kw)

    def precondition(self):
        K.kfac_precondition_batched(self.ctx, items=self._precond)

    def clip(self, max_norm, grad_scale=None):
        """What step() takes as grad_scale to clip the gradients by their global norm (which stays in self.norm): a device tensor, nothing waits."""
        K.kfac_grad_norm_batched(self.ctx, self._grads, self.norm, max_norm=max_norm, grad_scale=grad_scale, coef=self.coef)
        return self.coef

    def step(self, lr, grad_scale=None, **hyper):
        t = self.steps + 1
        K.kfac_adamw_batched(self.ctx, self._adamw, lr=lr, step=t, grad_scale=grad_scale, seed=self.seed if t > self.NEAREST_STEPS else 0, **hyper)
        self.steps = t


class RoutedExpertRunner(ExpertRunner):
    """A layer of experts behind its router, from tokens to tokens: logits (a layer of one expert, the router), each token's topk experts and their
    weights, tokens sorted by expert, the products, and the weighted sum of each token's results; and the way back.

    x is [tokens, d_in]; the sorted rows of a step stay in self.xs, the gradients of their results in self.gs, where update_factors() takes them.
    The router's parameters (fp32 [1, experts, d_in], no bias) take the optimizer step together with the experts'.  The logits are of the layer's type: in bf16
    two experts' often tie, and the lower one is chosen.
    """

    def __init__(self, experts, tokens, topk, d_in, d_out, normalize=True, bias=True, bf16=True, **kw):
        code = K.KFAC_BF16 if bf16 else K.KFAC_F32
        need = max(K.kfac_experts_dispatch_workspace_bytes(tokens, topk, experts), K.kfac_experts_workspace_bytes(1, tokens, d_in, experts, False, code),
                   K.kfac_grad_norm_workspace_bytes((K.kfac_grad_item * 2)(*(K.kfac_grad_item(n=experts * n) for n in (d_out * (d_in + 1), d_in)))))
        super().__init__(experts, tokens * topk, d_in, d_out, bias=bias, bf16=bf16, more_workspace=need, **kw)
        self.tokens, self.topk, self.normalize = tokens, topk, normalize
        f32, i32 = dict(dtype=torch.float32, device=self.dev), dict(dtype=torch.int32, device=self.dev)
        new = lambda *shape: torch.zeros(shape, dtype=self.dt, device=self.dev)  # noqa: E731
        self.router = torch.zeros((1, experts, d_in), **f32)
        self.router_weight = torch.zeros_like(self.router, dtype=self.dt) if bf16 else self.router
        self.router_grad = torch.zeros_like(self.router)
        self.router_state = self._state(self.router)
        self.logits, self.dlogits = new(tokens, experts), new(tokens, experts)
        self.ids, self.row = torch.zeros((tokens, topk), **i32), torch.zeros((tokens, topk), **i32)
        self.weights, self.dweights = torch.zeros((tokens, topk), **f32), torch.zeros((tokens, topk), **f32)
        self.all, self.offsets = torch.tensor([0, tokens], **i32), torch.zeros(experts + 1, **i32)
        self.xs, self.gs = new(tokens * topk, d_in), new(tokens * topk, d_out)
        self.out, self.dtokens = new(tokens, d_out), new(tokens, d_in)
        self._adamw = K.adamw_items([self._item(self.param, self.grad, self.state, self.weight),
                                     self._item(self.router, self.router_grad, self.router_state, self.router_weight)])
        self._grads = K.grad_items([self.grad, self.router_grad])
        self._masked = False                                 # whether the last forward() was given a mask

    def load(self, param, router):
        super().load(param)
        with own_stream(self, router):
            self.router.copy_(router)
            if self.router_weight is not self.router:
                self.router_weight.copy_(self.router)

    def forward(self, x, add=None, masked=None):
        """[tokens, d_out]: add (or zero) plus the weighted results of each token's experts.  masked: truth values [tokens, 1] (padding) or [tokens or 1, experts]
        (experts out of use) of what is not to be chosen; a token without a choice gets no result, and no gradient but what was added passes on, and whatever stands in
        a masked one's x and g (NaN among it) reaches nothing."""
        K.kfac_experts_forward(self.ctx, x, self.router_weight, self.all, self.logits)
        self._masked = masked is not None
        if self._masked:
            with own_stream(self, masked):
                self.logits.masked_fill_(masked, float("-inf"))
        K.kfac_experts_route(self.ctx, self.logits, self.ids, self.weights, normalize=self.normalize)
        K.kfac_experts_dispatch(self.ctx, self.ids, x, self.offsets, self.row, self.xs)
        super().forward(self.xs, self.offsets)
        K.kfac_experts_combine(self.ctx, self.y, self.row, self.weights, self.out, add=add)
        return self.out

    def backward(self, x, g, accumulate=False, gather=False):
        """The tokens' gradient (returned), every expert's (self.grad) and the router's (self.router_grad) from the output's.  (What was added passes g on.)
        gather: the sorted rows are made from x once more (where layers share self.xs, another's stand there by now)."""
        if gather:
            K.kfac_experts_gather(self.ctx, self.row, x, self.xs)
        K.kfac_experts_combine_grad(self.ctx, g, self.y, self.row, self.weights, self.gs, self.dweights)
        super().backward(self.xs, self.gs, self.offsets, accumulate=accumulate)
        K.kfac_experts_route_grad(self.ctx, self.logits, self.ids, self.dweights, self.dlogits, normalize=self.normalize)
        K.kfac_experts_input_grad(self.ctx, self.dlogits, self.router_weight, self.all, self.dtokens)
        if self._masked:                                     # (the logits of a padded token have no gradient, but zero times the NaN that may stand there is NaN)
            with own_stream(self, x):
                x = x.masked_fill(self.ids[:, :1] < 0, 0.0)
        K.kfac_experts_weight_grad(self.ctx, self.dlogits, x, self.all, self.router_grad, accumulate=accumulate)
        K.kfac_experts_combine(self.ctx, self.dx, self.row, None, self.dtokens, add=self.dtokens)
        return self.dtokens

    def update_factors(self, decay):
        super().update_factors(self.xs, self.gs, self.offsets, decay)
