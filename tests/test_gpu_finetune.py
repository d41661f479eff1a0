"""Training with orthogonalised momentum and adapters as the command runs them: the autograd function against differences and
the formulas, the optimiser against its own definition, and both commands for running."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2401_04044_b200 import Context, build
    build.build()
    c = Context(0)
    yield c
    c.close()


def layer(act, d, m, n, r, T, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    new = lambda s, *shape: (torch.randn(*shape, generator=g) * s).to(dtype).cuda()  # noqa: E731
    gated = act == "swiglu"
    W = {"W1": new(d ** -0.5, d, m), "W1u": new(d ** -0.5, d, m) if gated else None, "b1": None if gated else new(0.1, m),
         "W2": new(m ** -0.5, m, d), "b2": None if gated else new(0.1, d)}
    names = ["W1", "W2"] + (["W1u"] if gated else [])
    F = {k: (new(W[k].shape[0] ** -0.5, n, W[k].shape[0], r), new(0.3 * r ** -0.5, n, r, W[k].shape[1])) for k in names}
    index = torch.randint(-1, n, (T,), generator=g).to(torch.int32).cuda()
    return W, F, index, new(1.0, T, d), new(0.1, T, d)


def plain_ffn(act, X, W, F, index, scale):
    """The adapted layer in 64 bits from elementary operations."""
    f = lambda t: None if t is None else t.double()  # noqa: E731
    def side(x, name, b):  # noqa: E306
        A, B = F[name]
        y = x @ f(W[name]) + (0 if W.get(b) is None else f(W[b]))
        for i in range(A.shape[0]):
            y = y + ((index == i).double() * scale[i].double()).unsqueeze(1) * (x @ A[i] @ B[i])
        return y
    z = side(X, "W1", "b1")
    if act == "swiglu":
        h = z * torch.sigmoid(z) * side(X, "W1u", None)
    else:
        h = torch.nn.functional.gelu(z, approximate="none" if act == "gelu_erf" else "tanh")
    return side(h, "W2", "b2")


# bf16: Z, U, H, the activation's value and its gradient and each product's inner side are rounded on the way, seven roundings of
# an rms of 1.7e-3 at most each: 4.5e-3 with all of them, 8e-3 is asked for.  fp32: 1e-5 twice over.
@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 8e-3)])
@pytest.mark.parametrize("act,T", [("swiglu", 9), ("swiglu", 150), ("gelu_erf", 150), ("gelu_tanh", 33)])
def test_adapted_layer_and_its_gradients(ctx, act, T, dtype, tol):
    from paper_2401_04044_b200 import make_shape
    from paper_2401_04044_b200.train import adapted_ffn
    W, F, index, X, dY = layer(act, 64, 136, 3, 8, T, dtype)
    scale = torch.tensor([1.0, 0.5, 2.0], device="cuda")
    leaves = [X] + [t for v in F.values() for t in v]
    for t in leaves:
        t.requires_grad_()
    Y = adapted_ffn(ctx, make_shape(64, 136, act, dtype), X, W, F, index, scale)
    Y.backward(dY)
    ctx.poll()
    wide = {id(t): t.detach().double().requires_grad_() for t in leaves}
    ref = plain_ffn(act, wide[id(X)], W, {k: tuple(wide[id(t)] for t in v) for k, v in F.items()}, index, scale)
    ref.backward(dY.double())
    near = lambda a, b: float((a.double() - b).norm() / b.norm().clamp_min(1e-300))  # noqa: E731
    assert near(Y.detach(), ref.detach()) <= tol
    for t in leaves:
        assert near(t.grad, wide[id(t)].grad) <= tol


def test_gradients_of_a_projection_against_differences(ctx):
    from paper_2401_04044_b200 import Projection
    from paper_2401_04044_b200.train import adapted
    g = torch.Generator().manual_seed(3)
    new = lambda s, *shape: (torch.randn(*shape, generator=g) * s).cuda()  # noqa: E731
    p, T = Projection(24, 40, torch.float32), 13
    index = torch.randint(-1, 2, (T,), generator=g).to(torch.int32).cuda()
    tensors = {"X": new(1.0, T, 24), "A": new(0.2, 2, 24, 4), "B": new(0.5, 2, 4, 40), "base": new(1.0, T, 40)}
    C = new(1.0, T, 40)
    for t in tensors.values():
        t.requires_grad_()
    value = lambda X, A, B, base: float((adapted(ctx, p, X, A, B, index, base=base).double() * C.double()).sum())  # noqa: E731
    (adapted(ctx, p, tensors["X"], tensors["A"], tensors["B"], index, base=tensors["base"]) * C).sum().backward()
    for k, t in tensors.items():
        step = torch.randn(t.shape, generator=g).cuda()
        step = step / step.norm()
        with torch.no_grad():
            eps = 1e-2      # (the value is at most quadratic in each tensor: central differences are exact up to fp32's 1e-6 of it over eps)
            up, down = ({**tensors, k: t + s * eps * step} for s in (1, -1))
            slope = (value(**up) - value(**down)) / (2 * eps)
            assert abs(slope - float((t.grad.double() * step.double()).sum())) <= 2e-3 * max(1.0, float(t.grad.norm())), k


def test_frozen_tensors_may_not_ask_for_gradients(ctx):
    from paper_2401_04044_b200 import FFSplitError, Projection
    from paper_2401_04044_b200.train import Muon, adapted
    X, A, B = torch.randn(4, 8, device="cuda"), torch.randn(1, 8, 2, device="cuda"), torch.randn(1, 2, 8, device="cuda")
    index, W = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.randn(8, 8, device="cuda", requires_grad=True)
    with pytest.raises(FFSplitError):
        adapted(ctx, Projection(8, 8, torch.float32), X, A, B, index, W=W)
    with torch.no_grad():
        adapted(ctx, Projection(8, 8, torch.float32), X, A, B, index, W=W.detach())
    with pytest.raises(FFSplitError):
        Muon(ctx, [torch.zeros(8, device="cuda", requires_grad=True)])


def test_optimiser_steps_matrices_and_stacks(ctx):
    from paper_2401_04044_b200.train import Muon
    g = torch.Generator().manual_seed(1)
    P = [torch.randn(*s, generator=g).cuda().requires_grad_() for s in ((40, 100), (3, 70, 16), (2, 3, 90, 80))]
    start = [p.detach().clone() for p in P]
    opt = Muon(ctx, P, lr=0.1, weight_decay=0.5)
    momenta = [torch.zeros_like(p).double() for p in P]
    ref = [p.detach().double() for p in P]
    for k in range(3):
        for p, m, r in zip(P, momenta, ref):
            p.grad = torch.randn(p.shape, generator=g).cuda()
            G = p.grad.double()
            m.mul_(0.95).add_(G)
            for idx in np.ndindex(*p.shape[:-2]):
                u = (G + 0.95 * m)[idx]
                x = u / u.norm()
                for _ in range(5):
                    s = x @ x.T
                    x = 3.4445 * x + (-4.7750 * s + 2.0315 * (s @ s)) @ x
                r[idx] = (1 - 0.1 * 0.5) * r[idx] - 0.1 * 0.2 * math.sqrt(max(u.shape)) * x
        opt.step()
        opt.zero_grad()
    ctx.poll()
    for p, r, s in zip(P, ref, start):
        assert not torch.equal(p.detach(), s)
        assert float((p.detach().double() - r).norm() / r.norm()) <= 3e-5      # three steps of 1e-5 each
    opt.step()      # without gradients: nothing


@pytest.mark.parametrize("argv", [["--optimizer", "muon"], ["--optimizer", "muon", "--act", "gelu_erf"], ["--adapters", "8"], ["--adapters", "16", "--act", "gelu_tanh"]])
def test_command_runs(argv, capsys):
    from paper_2401_04044_b200 import train
    train.main(["--d", "64", "--m", "160", "--tokens", "96", "--steps", "3", *argv])
    assert "loss" in capsys.readouterr().out
