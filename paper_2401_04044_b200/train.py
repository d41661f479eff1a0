"""Training a feed-forward layer with the library's kernels, from PyTorch.

`ffn` is the layer as an autograd function (ffsplit_train_forward / ffsplit_train_backward), `clip_grad_norm_` the
global gradient norm and clipping (ffsplit_grad_clip).  Run as a command,

    python -m paper_2401_04044_b200.train [--d 1024 --m 2752 --act swiglu --tokens 512 --steps 30]

it starts from a layer whose weights were rounded to eight levels, fine-tunes it towards the outputs of the layer it
was rounded from, and takes the result through the library's own path: score, select, pack, forward.
"""
from __future__ import annotations

import argparse
from typing import Iterable, Optional, Union

import torch
from torch.autograd.function import once_differentiable

from .binding import Context, GradList, Shape, make_shape


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
    return norm


def _eight_levels(w: torch.Tensor) -> torch.Tensor:
    """Rounded to nearest on eight levels between the smallest and the largest value of each column."""
    lo, hi = w.float().amin(0, keepdim=True), w.float().amax(0, keepdim=True)
    step = (hi - lo) / 7
    return (lo + torch.round((w.float() - lo) / step) * step).to(w.dtype)


def finetune(lib: Context, d: int, m: int, act: str = "swiglu", tokens: int = 512, steps: int = 30, lr: float = 5.0,
             max_norm: float = 0.05, dtype=torch.bfloat16, seed: int = 0, report=None):
    """Recovers a layer whose weights were rounded to eight levels: SGD on the mean squared distance between its outputs and
    those of the layer before rounding.  -> (losses, the layer's shape, its weights as a dict)"""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda scale, *s: (torch.randn(*s, generator=gen, device="cuda") * scale).to(dtype)  # noqa: E731
    gated = act == "swiglu"
    shape = make_shape(d, m, act, dtype)
    whole = {"W1": new(d ** -0.5, d, m), "W1u": new(d ** -0.5, d, m) if gated else None, "b1": None if gated else new(0.1, m),
             "W2": new(m ** -0.5, m, d), "b2": None if gated else new(0.1, d)}
    P = {k: None if v is None else (_eight_levels(v) if v.dim() == 2 else v.clone()).requires_grad_() for k, v in whole.items()}
    params = [v for v in P.values() if v is not None]
    master = [p.detach().float() for p in params]      # 32-bit copies: a bf16 step this small would be rounded away
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
            for p, w in zip(params, master):
                w.add_(p.grad.float(), alpha=-lr)
                p.copy_(w)
                p.grad = None
        losses.append(loss.item())
        if report:
            report(step, losses[-1], norm.item())
    lib.poll()
    return losses, shape, {k: None if v is None else v.detach() for k, v in P.items()}


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--d", type=int, default=1024)
    ap.add_argument("--m", type=int, default=2752)
    ap.add_argument("--act", default="swiglu", choices=["swiglu", "gelu_erf", "gelu_tanh"])
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--lr", type=float, default=5.0)
    a = ap.parse_args(argv)
    lib = Context(0)
    losses, shape, W = finetune(lib, a.d, a.m, a.act, a.tokens, a.steps, a.lr,
                                report=lambda i, l, n: print(f"step {i:3d}  loss {l:.5f}  gradient norm {n:.4f}"))
    # the tuned layer, split: a tenth of its neurons kept, the others left out
    T, m = 512, shape.m
    k = m // 10
    lib.ensure_workspace(max(lib.workspace_size(shape, T, T, k, 0), lib.workspace_size(shape, T, T, m, 0)))
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
