"""Training a feed-forward layer with the library's kernels, from PyTorch.

`ffn` is the layer as an autograd function (ffsplit_train_forward / ffsplit_train_backward), `clip_grad_norm_` the
global gradient norm and clipping (ffsplit_grad_clip), `Muon` an optimiser for matrices (ffsplit_muon_step), `adapted` a
projection with low-rank adapters (ffsplit_adapter_forward / ffsplit_adapter_backward).  Run as a command,

    python -m paper_2401_04044_b200.train [--d 1024 --m 2752 --act swiglu --tokens 512 --steps 30 --optimizer muon --adapters 16]

it starts from a layer whose weights were rounded to eight levels, fine-tunes it towards the outputs of the layer it
was rounded from, and takes the result through the library's own path: score, select, pack, forward.  With --adapters R
the rounded weights stay as they are and rank-R adapters beside them are trained instead, two in one batch.
"""
from __future__ import annotations

import argparse
import math
from typing import Iterable, Optional, Union

import torch
from torch.autograd.function import once_differentiable

from .binding import Context, FFSplitError, GradList, MuonList, Projection, Shape, make_shape


class _FFN(torch.autograd.Function):
    @staticmethod
    def forward(ctx, lib: Context, shape: Shape, grad_mode: bool, X, W1, W1u, b1, W2, b2):
        T = X.shape[0]
        saved_bytes, workspace = lib.train_sizes(shape, T)
        lib.ensure_workspace(workspace)
        keep = grad_mode and any(ctx.needs_input_grad)
        saved = torch.empty(saved_bytes, dtype=torch.uint8, device=X.device) if keep else None
        Y = torch.empty_like(X)
        lib.train_forward(shape, W1, b1, W2, b2, X, Y, saved=saved, W1u=W1u)
        ctx.lib, ctx.shape, ctx.has = lib, shape, (W1u is not None, b1 is not None, b2 is not None)
        ctx.save_for_backward(X, W1, W1u, W2, saved)
        return Y

    @staticmethod
    @once_differentiable
    def backward(ctx, dY):
        X, W1, W1u, W2, saved = ctx.saved_tensors
        lib, shape = ctx.lib, ctx.shape
        lib.ensure_workspace(lib.train_sizes(shape, X.shape[0])[1])
        _, _, _, need_X, need_W1, need_W1u, need_b1, need_W2, need_b2 = ctx.needs_input_grad
        new = lambda need, *dims: torch.empty(dims, dtype=X.dtype, device=X.device) if need else None  # noqa: E731
        d, m = shape.d, shape.m
        g = {"dX": new(need_X, *X.shape), "dW1": new(need_W1, d, m), "dW1u": new(need_W1u and ctx.has[0], d, m),
             "db1": new(need_b1 and ctx.has[1], m), "dW2": new(need_W2, m, d), "db2": new(need_b2 and ctx.has[2], d)}
        # (what autograd hands over may be expanded, or a piece of a larger gradient that starts anywhere)
        dY = dY.contiguous()
        if dY.data_ptr() % 16:
            dY = dY.clone()
        lib.train_backward(shape, W1, None, W2, X, saved, dY, W1u=W1u, **g)
        return None, None, None, g["dX"], g["dW1"], g["dW1u"], g["db1"], g["dW2"], g["db2"]


def ffn(lib: Context, shape: Shape, X, W1, W2, b1=None, b2=None, W1u=None) -> torch.Tensor:
    """act(X W1 + b1) W2 + b2, or (SiLU(X W1) * (X W1u)) W2 + b2, differentiable once in X and the weights.  X [T, d] and
    the weights are contiguous tensors of the layer's type on the context's device; the calls run on the current stream.
    Where the context's workspace is too small for T tokens it is replaced, which waits for the device and is refused while a
    graph is captured (lib.ensure_workspace(lib.train_sizes(shape, T)[1]) does it before).  Calls on one context share its
    workspace: they may not overlap on the GPU, whatever their streams."""
    return _FFN.apply(lib, shape, torch.is_grad_enabled(), X, W1, W1u, b1, W2, b2)


def clip_grad_norm_(lib: Context, parameters: Union[torch.Tensor, Iterable[torch.Tensor]], max_norm: float,
                    norm: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Scales the parameters' gradients in place so that their norm is at most max_norm; returns the norm (float32[1] on
    the device, not waited for).  A parameter that is named twice counts once.  A non-finite norm leaves the gradients as
    they are and is reported by lib.poll().  Workspace and streams: as for ffn()."""
    parameters = [parameters] if isinstance(parameters, torch.Tensor) else parameters
    grads = [p.grad for p in {id(p): p for p in parameters}.values() if p.grad is not None]
    if norm is None:
        norm = torch.empty(1, dtype=torch.float32, device=f"cuda:{lib.device}")
    lib.ensure_workspace(lib.grad_workspace_size(len(grads)))
    lib.clip_grads(GradList(lib.device, grads), max_norm, norm)
    for g in grads:      # (written by address: see Muon.step)
        torch.autograd.graph.increment_version(g)
    return norm


def _matrices(t: torch.Tensor):
    """The matrices of a parameter: itself, or one to each leading index (a stack of adapters' factors)."""
    return [t] if t.dim() == 2 else list(t.view(-1, *t.shape[-2:]))      # (a view: what is updated is the parameter itself)


class Muon(torch.optim.Optimizer):
    """Momentum, orthogonalised, as the update of matrices (ffsplit_muon_step): W <- (1 - lr weight_decay) W - lr 0.2
    sqrt(max(rows, cols)) X, where X is the orthogonal factor of the momentum and 0.2 sqrt(...) makes its elements as large as
    0.2 in the mean.  Parameters are contiguous, float32 or bfloat16, with two dimensions, or more (a matrix to each leading
    index); momentum is float32.  All matrices of a group are one call on the current stream; a gradient that is not finite leaves its
    matrix alone and is reported by lib.poll().  Workspace and streams: as for ffn()."""

    def __init__(self, lib: Context, params, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                 coefficients=None, iterations: int = 5):
        self.lib = lib
        super().__init__(params, dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, coefficients=coefficients,
                                      iterations=iterations))

    def add_param_group(self, param_group):
        super().add_param_group(param_group)
        fits = lambda p: p.dim() >= 2 and p.dtype in (torch.float32, torch.bfloat16) and p.numel() > 0 and p.is_contiguous()  # noqa: E731
        if not all(fits(p) for p in self.param_groups[-1]["params"]):
            self.param_groups.pop()
            raise FFSplitError(2, "Muon", "parameters are contiguous float32 or bfloat16 matrices, or stacks of them, and not empty")

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)
        # (which gives a state its parameter's type: momentum is float32 beside bfloat16 parameters too)
        saved = [i for group in state_dict["param_groups"] for i in group["params"]]
        for i, p in zip(saved, (p for group in self.param_groups for p in group["params"])):
            if "momentum" in state_dict["state"].get(i, {}):
                self.state[p]["momentum"] = state_dict["state"][i]["momentum"].to(p.device, torch.float32, copy=True)

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        steps = []      # all of them are looked at before one is taken
        for group in self.param_groups:
            params = [p for p in group["params"] if p.grad is not None]
            if not params:
                continue
            for p in params:
                if "momentum" not in self.state[p]:
                    self.state[p]["momentum"] = torch.zeros(p.shape, dtype=torch.float32, device=p.device)
            each = lambda tensors: [m for t in tensors for m in _matrices(t)]  # noqa: E731
            W = each(params)
            rates = [group["lr"] * 0.2 * math.sqrt(max(w.shape)) for w in W]
            tensors = MuonList(self.lib.device, each(p.grad.contiguous() for p in params), W, each(self.state[p]["momentum"] for p in params),
                               rates, group["lr"] * group["weight_decay"])
            steps.append((group, params, tensors))
        if steps:
            self.lib.ensure_workspace(max(self.lib.muon_workspace_size(tensors) for _, _, tensors in steps))
        for group, params, tensors in steps:
            self.lib.muon_step(tensors, group["momentum"], group["nesterov"], group["coefficients"], group["iterations"])
            for p in params:      # (the library writes by address: a graph that still holds a parameter must not go on with its new value)
                torch.autograd.graph.increment_version(p)
        return loss


class _Adapted(torch.autograd.Function):
    @staticmethod
    def forward(ctx, lib: Context, p: Projection, X, A, B, index, W, b, base, scale):
        if any(ctx.needs_input_grad[i] for i in (6, 7, 9)):
            raise FFSplitError(1, "adapted", "W, b and scale stay as they are: they cannot require gradients here")
        lib.ensure_workspace(lib.adapter_workspace_size(p, A.shape[0], A.shape[2], X.shape[0]))
        Y = torch.empty(X.shape[0], p.outer, dtype=X.dtype, device=X.device)
        lib.adapter_forward(p, X, A, B, index, Y, W=W, b=b, base=base, scale=scale)
        ctx.lib, ctx.p = lib, p
        ctx.save_for_backward(X, A, B, index, W, scale)
        return Y

    @staticmethod
    @once_differentiable
    def backward(ctx, dY):
        X, A, B, index, W, scale = ctx.saved_tensors
        lib, p = ctx.lib, ctx.p
        lib.ensure_workspace(lib.adapter_workspace_size(p, A.shape[0], A.shape[2], X.shape[0]))
        # (what autograd hands over may be expanded, or a piece of a larger gradient that starts anywhere)
        dY = dY.contiguous()
        if dY.data_ptr() % 16:
            dY = dY.clone()
        new = lambda i, t: torch.empty_like(t) if ctx.needs_input_grad[i] else None  # noqa: E731
        g = {"dX": new(2, X), "dA": new(3, A), "dB": new(4, B)}
        if any(v is not None for v in g.values()):
            lib.adapter_backward(p, X, A, B, index, dY, W=W, scale=scale, **g)
        return None, None, g["dX"], g["dA"], g["dB"], None, None, None, dY if ctx.needs_input_grad[8] else None, None


def adapted(lib: Context, projection: Projection, X, A, B, index, W=None, b=None, base=None, scale=None) -> torch.Tensor:
    """(X W + b, or base, or nothing) + scale_i (X A_i) B_i with i = index[t] (negative: none), differentiable once in X, A,
    B and base.  X [T, inner], A [n, inner, r], B [n, r, outer], index int32 [T], scale float32 [n].  Workspace and streams:
    as for ffn()."""
    return _Adapted.apply(lib, projection, X, A, B, index, W, b, base, scale)


def adapted_ffn(lib: Context, shape: Shape, X, weights: dict, factors: dict, index, scale=None) -> torch.Tensor:
    """The layer with an adapter beside each of its projections: factors holds (A, B) under "W1", "W2" and, of gated layers,
    "W1u"; weights as finetune() has them."""
    dt, w = X.dtype, weights
    up, down = Projection(shape.d, shape.m, dt), Projection(shape.m, shape.d, dt)
    side = lambda p, x, name, b: adapted(lib, p, x, *factors[name], index, W=w[name], b=w[b] if b else None, scale=scale)  # noqa: E731
    Z = side(up, X, "W1", "b1")
    if shape.act == 2:
        H = torch.nn.functional.silu(Z) * side(up, X, "W1u", None)
    else:
        H = torch.nn.functional.gelu(Z, approximate="none" if shape.act == 0 else "tanh")
    return side(down, H, "W2", "b2")


def _eight_levels(w: torch.Tensor) -> torch.Tensor:
    """Rounded to nearest on eight levels between the smallest and the largest value of each column."""
    lo, hi = w.float().amin(0, keepdim=True), w.float().amax(0, keepdim=True)
    step = (hi - lo) / 7
    return (lo + torch.round((w.float() - lo) / step) * step).to(w.dtype)


def finetune(lib: Context, d: int, m: int, act: str = "swiglu", tokens: int = 512, steps: int = 30, lr: float = 5.0,
             max_norm: float = 0.05, dtype=torch.bfloat16, seed: int = 0, report=None, optimizer: str = "sgd"):
    """Recovers a layer whose weights were rounded to eight levels: SGD, or orthogonalised momentum ("muon"; lr is then the step
    of its matrices, biases take SGD), on the mean squared distance between its outputs and those of the layer before
    rounding.  -> (losses, the layer's shape, its weights as a dict)"""
    if optimizer not in ("sgd", "muon"):
        raise ValueError(f"unknown optimizer {optimizer!r}: sgd or muon")
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda scale, *s: (torch.randn(*s, generator=gen, device="cuda") * scale).to(dtype)  # noqa: E731
    gated = act == "swiglu"
    shape = make_shape(d, m, act, dtype)
    whole = {"W1": new(d ** -0.5, d, m), "W1u": new(d ** -0.5, d, m) if gated else None, "b1": None if gated else new(0.1, m),
             "W2": new(m ** -0.5, m, d), "b2": None if gated else new(0.1, d)}
    P = {k: None if v is None else (_eight_levels(v) if v.dim() == 2 else v.clone()).requires_grad_() for k, v in whole.items()}
    params = [v for v in P.values() if v is not None]
    master = [p.detach().float() for p in params]      # 32-bit copies: a bf16 step this small would be rounded away
    matrices = [i for i, p in enumerate(params) if optimizer == "muon" and p.dim() == 2]
    momenta = [torch.zeros_like(master[i]) for i in matrices]
    run = lambda X, w: ffn(lib, shape, X, w["W1"], w["W2"], w["b1"], w["b2"], w["W1u"])  # noqa: E731
    losses = []
    for step in range(steps):
        X = new(1.0, tokens, d)
        with torch.no_grad():
            target = run(X, whole)
        loss = (run(X, P).float() - target.float()).square().mean()
        loss.backward()
        norm = clip_grad_norm_(lib, params, max_norm)
        with torch.no_grad():
            if matrices:
                tensors = lib.muon_list([master[i] for i in matrices], [params[i].grad for i in matrices], momenta,
                                        [lr * 0.2 * math.sqrt(max(master[i].shape)) for i in matrices])
                lib.ensure_workspace(lib.muon_workspace_size(tensors))
                lib.muon_step(tensors)
            for i, (p, w) in enumerate(zip(params, master)):
                if i not in matrices:
                    w.add_(p.grad.float(), alpha=-(lr if optimizer == "sgd" else 5.0))
                p.copy_(w)
                p.grad = None
        losses.append(loss.item())
        if report:
            report(step, losses[-1], norm.item())
    lib.poll()
    return losses, shape, {k: None if v is None else v.detach() for k, v in P.items()}


def finetune_adapters(lib: Context, d: int, m: int, act: str = "swiglu", rank: int = 16, tokens: int = 512, steps: int = 30, lr: float = 2e-2,
                      dtype=torch.bfloat16, seed: int = 0, report=None):
    """Two tasks beside one layer whose weights were rounded to eight levels and stay so: each has adapters of its own, trained
    in one batch (half of the tokens each) towards the layer before rounding, in the second task with a rank-4 change of its W2.
    -> (losses, the layer's shape, its weights, the factors)"""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda scale, *s: (torch.randn(*s, generator=gen, device="cuda") * scale).to(dtype)  # noqa: E731
    gated = act == "swiglu"
    shape = make_shape(d, m, act, dtype)
    whole = {"W1": new(d ** -0.5, d, m), "W1u": new(d ** -0.5, d, m) if gated else None, "b1": None if gated else new(0.1, m),
             "W2": new(m ** -0.5, m, d), "b2": None if gated else new(0.1, d)}
    W = {k: _eight_levels(v) if v is not None and v.dim() == 2 else v for k, v in whole.items()}
    changed = whole["W2"] + new(m ** -0.5, m, 4) @ new(1.0, 4, d)
    names = ["W1", "W2"] + (["W1u"] if gated else [])
    factors = {}
    for k in names:
        inner, outer = W[k].shape
        factors[k] = tuple(t.requires_grad_() for t in (new(inner ** -0.5, 2, inner, rank), torch.zeros(2, rank, outer, dtype=dtype, device="cuda")))
    params = [t for k in names for t in factors[k]]
    opt = Muon(lib, params, lr=lr)
    index = (torch.arange(tokens, device="cuda") * 2 // tokens).to(torch.int32)
    losses = []
    for step in range(steps):
        X = new(1.0, tokens, d)
        with torch.no_grad():
            first, second = (ffn(lib, shape, X, whole["W1"], W2, whole["b1"], whole["b2"], whole["W1u"]) for W2 in (whole["W2"], changed))
            target = torch.where((index == 0).unsqueeze(1), first, second)
        loss = (adapted_ffn(lib, shape, X, W, factors, index).float() - target.float()).square().mean()
        loss.backward()
        norm = clip_grad_norm_(lib, params, math.inf)
        opt.step()
        opt.zero_grad()
        losses.append(loss.item())
        if report:
            report(step, losses[-1], norm.item())
    lib.poll()
    return losses, shape, W, {k: tuple(t.detach() for t in v) for k, v in factors.items()}


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--d", type=int, default=1024)
    ap.add_argument("--m", type=int, default=2752)
    ap.add_argument("--act", default="swiglu", choices=["swiglu", "gelu_erf", "gelu_tanh"])
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--optimizer", default="sgd", choices=["sgd", "muon"])
    ap.add_argument("--adapters", type=int, default=0, metavar="RANK")
    ap.add_argument("--lr", type=float, default=None, help="5 (sgd), 0.001 (muon), 0.02 (adapters)")
    a = ap.parse_args(argv)
    lr = a.lr if a.lr is not None else 2e-2 if a.adapters else 5.0 if a.optimizer == "sgd" else 1e-3
    lib = Context(0)
    report = lambda i, l, n: print(f"step {i:3d}  loss {l:.5f}  gradient norm {n:.4f}")  # noqa: E731
    if a.adapters:
        losses, _, _, factors = finetune_adapters(lib, a.d, a.m, a.act, a.adapters, a.tokens, a.steps, lr, report=report)
        print(f"loss {losses[0]:.5f} -> {losses[-1]:.5f}; two adapters of {sum(t[0].numel() for v in factors.values() for t in v)} elements each")
        return
    losses, shape, W = finetune(lib, a.d, a.m, a.act, a.tokens, a.steps, lr, optimizer=a.optimizer, report=report)
    # the tuned layer, split: a tenth of its neurons kept, the others left out
    T, m = 512, shape.m
    k = m // 10
    lib.ensure_workspace(max(lib.workspace_size(shape, T, T, k, 0), lib.workspace_size(shape, T, T, m, 0), lib.train_sizes(shape, T)[1]))
    X = torch.randn(T, a.d, device="cuda").to(torch.bfloat16)
    energy, scores = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    lib.score(shape, W["W1"], W["b1"], W["W2"], X, energy, scores, W1u=W["W1u"])
    heavy = torch.empty(k, dtype=torch.int32, device="cuda")
    lib.select(scores, k, heavy)
    blob = torch.empty(lib.pack_size(shape, k, 0)[0], dtype=torch.uint8, device="cuda")
    lib.pack(shape, W["W1"], W["b1"], W["W2"], W["b2"], heavy, k, None, blob, W1u=W["W1u"])
    Y, full = torch.empty_like(X), torch.empty_like(X)
    lib.forward(blob, X, Y)
    lib.train_forward(shape, W["W1"], W["b1"], W["W2"], W["b2"], X, full, W1u=W["W1u"])
    lib.poll()
    off = float((Y.float() - full.float()).norm() / full.float().norm())
    print(f"loss {losses[0]:.5f} -> {losses[-1]:.5f}; the {k} heaviest of {m} neurons alone are {off:.3f} off the layer's output")


if __name__ == "__main__":
    main()
