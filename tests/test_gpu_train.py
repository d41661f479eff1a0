"""Training calls (forward with what the backward needs, backward, gradient norm and clipping) against plain
implementations in 64 bits, on the same stored inputs.

Tolerances.  bf16 layers: an output passes at most three roundings to bf16 on its way (the hidden matrix or its
gradient, the factor it was formed from, itself), each at most 2^-9 relative and independent of the others:
sqrt(3) 2^-9 = 3.4e-3 of the norm, with the 20 kept bits of G and U and the approximate exponentials below 2e-4:
4e-3.  fp32 layers: the library's 1e-5.  Single elements: a sum of n terms may cancel, so they are held to
8 times that bound of the largest element."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

NORM_TOL = {"bf16": 4e-3, "f32": 1e-5}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ctx():
    from paper_2401_04044_b200 import Context, build
    build.build()
    c = Context(0)
    c.ensure_workspace(1 << 20)
    yield c
    c.close()


def act64(z, act):
    if act == "swiglu":
        s = 1 / (1 + np.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    if act == "gelu_erf":
        phi = torch.special.ndtr(torch.from_numpy(z)).numpy()
        return z * phi, phi + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c, a = math.sqrt(2 / math.pi), 0.044715
    t = np.tanh(c * (z + a * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * a * z * z)


def ffn64(L, act):
    """Forward and backward of one layer in 64 bits; L holds numpy arrays (None where the layer has no such tensor)."""
    z = L["X"] @ L["W1"] + (0 if L["b1"] is None else L["b1"])
    a, s = act64(z, act)
    u = None if L["W1u"] is None else L["X"] @ L["W1u"]
    h = a if u is None else a * u
    dh = L["dY"] @ L["W2"].T
    dz = dh * s if u is None else dh * s * u
    r = {"Y": h @ L["W2"] + (0 if L["b2"] is None else L["b2"]), "dX": dz @ L["W1"].T, "dW1": L["X"].T @ dz,
         "dW2": h.T @ L["dY"], "db2": L["dY"].sum(0)}
    if u is not None:
        r["dX"] = r["dX"] + (dh * a) @ L["W1u"].T
        r["dW1u"] = L["X"].T @ (dh * a)
    else:
        r["db1"] = dz.sum(0)
    return r


def draw(act, dtype, d, m, T, seed=0, b1=True, b2=True, scale=1.0):
    g = torch.Generator().manual_seed(1000 * seed + d + 7 * m + 13 * T)
    new = lambda s, *shape: (torch.randn(*shape, generator=g) * s).to(DT[dtype])  # noqa: E731
    gated = act == "swiglu"
    w = 1.3 / math.sqrt(d)
    return {"X": new(scale, T, d), "W1": new(w, d, m), "W1u": new(w, d, m) if gated else None,
            "b1": new(0.2, m) if b1 and not gated else None, "W2": new(1 / math.sqrt(m), m, d),
            "b2": new(0.2, d) if b2 else None, "dY": new(0.01, T, d)}


def guarded(shape, dt):
    """An output tensor with 32 elements on either side that a call must not touch."""
    n = int(np.prod(shape))
    room = (n + 63) // 32 * 32 + 64
    flat = torch.full((room,), -7.0, dtype=dt, device="cuda")
    return flat, flat[32:32 + n].view(*shape)


def run(ctx, L, act, dtype, want=("dX", "dW1", "dW1u", "db1", "dW2", "db2"), keep=True, stream=None):
    import paper_2401_04044_b200 as ff
    D = {k: None if v is None else v.cuda() for k, v in L.items()}
    (T, d), m = L["X"].shape, L["W1"].shape[1]
    shape = ff.make_shape(d, m, act, DT[dtype])
    saved_bytes, ws = ctx.train_sizes(shape, T)
    ctx.ensure_workspace(ws)
    saved = torch.full((saved_bytes,), 0xFF, dtype=torch.uint8, device="cuda") if keep else None
    bufs = {"Y": guarded((T, d), DT[dtype])}
    gated = act == "swiglu"
    for k, s in {"dX": (T, d), "dW1": (d, m), "dW1u": (d, m), "db1": (m,), "dW2": (m, d), "db2": (d,)}.items():
        if k in want and not (gated and k == "db1") and not (not gated and k == "dW1u"):
            bufs[k] = guarded(s, DT[dtype])
    torch.cuda.synchronize()
    ctx.train_forward(shape, D["W1"], D["b1"], D["W2"], D["b2"], D["X"], bufs["Y"][1], saved=saved, W1u=D["W1u"], stream=stream)
    if keep:
        ctx.train_backward(shape, D["W1"], D["b1"], D["W2"], D["X"], saved, D["dY"], W1u=D["W1u"], stream=stream,
                           **{k: v[1] for k, v in bufs.items() if k != "Y"})
    ctx.poll(stream)
    torch.cuda.synchronize()
    for k, (flat, t) in bufs.items():
        assert (flat[:32] == -7).all() and (flat[32 + t.numel():] == -7).all(), f"{k}: written outside the tensor"
        if not keep and k != "Y":
            assert (t == -7).all()
    return {k: t.cpu() for k, (_, t) in bufs.items() if keep or k == "Y"}


def check(got, L, act, dtype, names=None):
    ref = ffn64({k: None if v is None else v.double().numpy() for k, v in L.items()}, act)
    for k, v in got.items():
        if names and k not in names:
            continue
        x, r = v.double().numpy(), ref[k]
        norm = np.linalg.norm(r)
        err = np.linalg.norm(x - r) / norm if norm else np.linalg.norm(x)
        big = np.abs(x - r).max() / max(np.abs(r).max(), 1e-300)
        tol = NORM_TOL[dtype]
        assert err <= tol and big <= 8 * tol, f"{k}: {err:.2e} of the norm (<= {tol}), {big:.2e} of the largest element"


SHAPES = [
    ("bf16", 8, 1, 1), ("bf16", 64, 7, 3), ("bf16", 136, 130, 129), ("bf16", 256, 1024, 64), ("bf16", 520, 771, 257),
    ("bf16", 1024, 264, 1), ("bf16", 72, 2056, 1000), ("bf16", 264, 96, 515), ("bf16", 648, 1288, 20),
    ("f32", 1, 1, 1), ("f32", 33, 65, 31), ("f32", 130, 257, 300), ("f32", 256, 512, 2), ("f32", 515, 130, 129),
]


@pytest.mark.parametrize("act", ["swiglu", "gelu_erf", "gelu_tanh"])
@pytest.mark.parametrize("dtype,d,m,T", SHAPES)
def test_forward_and_backward(ctx, dtype, d, m, T, act):
    L = draw(act, dtype, d, m, T)
    check(run(ctx, L, act, dtype), L, act, dtype)


@pytest.mark.parametrize("dtype,act,d,m,T", [("bf16", "swiglu", 1024, 2816, 2000), ("bf16", "gelu_erf", 2048, 1000, 1500),
                                             ("f32", "swiglu", 640, 1111, 1000)])
def test_many_tiles(ctx, dtype, act, d, m, T):
    L = draw(act, dtype, d, m, T, seed=3)
    check(run(ctx, L, act, dtype), L, act, dtype)


@pytest.mark.parametrize("dtype,act,b1,b2", [("bf16", "gelu_erf", False, True), ("f32", "gelu_tanh", True, False),
                                             ("bf16", "swiglu", False, False), ("f32", "gelu_erf", False, False)])
def test_layers_without_biases(ctx, dtype, act, b1, b2):
    L = draw(act, dtype, 72, 200, 50, b1=b1, b2=b2)
    check(run(ctx, L, act, dtype), L, act, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["swiglu", "gelu_erf"])
def test_each_gradient_alone_and_nothing_kept(ctx, dtype, act):
    L = draw(act, dtype, 136, 200, 150)
    whole = run(ctx, L, act, dtype)
    for k in whole:
        if k == "Y":
            part = run(ctx, L, act, dtype, keep=False)
        else:
            part = run(ctx, L, act, dtype, want=(k,))
        assert torch.equal(part[k], whole[k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_again_and_on_another_stream(ctx, dtype):
    L = draw("swiglu", dtype, 264, 700, 333)
    a, b = run(ctx, L, "swiglu", dtype), run(ctx, L, "swiglu", dtype)
    c = run(ctx, L, "swiglu", dtype, stream=torch.cuda.Stream())
    for k in a:
        assert torch.equal(a[k], b[k]) and torch.equal(a[k], c[k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["swiglu", "gelu_erf", "gelu_tanh"])
def test_saturated_activations(ctx, dtype, act):
    """Pre-activations far out on both sides: the activation is 0 or the identity there, its slope 0 or 1."""
    L = draw(act, dtype, 64, 96, 70, scale=60.0)
    got = run(ctx, L, act, dtype)
    assert all(torch.isfinite(v).all() for v in got.values())
    check(got, L, act, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-12, 1e12])
def test_scale_of_the_gradient(ctx, dtype, scale):
    """The backward pass is linear in dY, over many orders of magnitude."""
    L = draw("swiglu", dtype, 64, 130, 90)
    L["dY"] = (L["dY"].double() * scale).to(DT[dtype])
    check(run(ctx, L, "swiglu", dtype), L, "swiglu", dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zero_inputs(ctx, dtype):
    L = draw("swiglu", dtype, 64, 100, 40)
    L["X"].zero_()
    got = run(ctx, L, "swiglu", dtype)
    assert (got["dX"] == 0).all() and (got["dW1"] == 0).all() and (got["dW2"] == 0).all()
    assert torch.equal(got["Y"], L["b2"].expand(40, 64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_non_finite_token_stays_in_its_row(ctx, dtype, bad):
    T = 150
    L = draw("swiglu", dtype, 72, 100, T)
    clean = run(ctx, L, "swiglu", dtype)
    L["X"][77, 5] = bad
    got = run(ctx, L, "swiglu", dtype)
    rest = [t for t in range(T) if t != 77]
    for k in ("Y", "dX"):
        assert torch.equal(got[k][rest], clean[k][rest])
        assert not torch.isfinite(got[k][77]).any()
    assert not torch.isfinite(got["dW1"][5]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["gelu_erf", "gelu_tanh"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_non_finite_token_of_a_gelu_layer_stays_in_its_row(ctx, dtype, act, bad):
    T = 150
    L = draw(act, dtype, 72, 100, T)
    clean = run(ctx, L, act, dtype)
    L["X"][77, 5] = bad
    got = run(ctx, L, act, dtype)
    rest = [t for t in range(T) if t != 77]
    for k in ("Y", "dX"):
        assert torch.equal(got[k][rest], clean[k][rest])
        assert not torch.isfinite(got[k][77]).any()
    assert not torch.isfinite(got["dW1"][5]).any()
    assert torch.equal(got["db2"], clean["db2"])


@pytest.mark.parametrize("dtype,act,d,m", [("bf16", "swiglu", 4096, 11008), ("bf16", "gelu_tanh", 5120, 20480), ("bf16", "swiglu", 1000, 2731),
                                           ("f32", "gelu_erf", 2048, 4097)])
@pytest.mark.parametrize("T", [1, 2, 7, 33])
def test_few_tokens_through_wide_layers(ctx, dtype, act, d, m, T):
    D = draw_on_the_device(act, dtype, d, m, T)
    check_on_the_device(run(ctx, D, act, dtype), D, act, dtype)


def test_bias_gradients_of_a_very_wide_layer(ctx):
    """More blocks of columns for db1 than there are tickets, while db2's rows are cut."""
    import paper_2401_04044_b200 as ff
    d, m, T = 8, 530_000, 520
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda s, *dims: (torch.randn(*dims, generator=g, device="cuda") * s).bfloat16()  # noqa: E731
    X, W1, W2, dY = new(1.0, T, d), new(0.3, d, m), new(0.01, m, d), new(0.01, T, d)
    shape = ff.make_shape(d, m, "gelu_tanh", torch.bfloat16)
    saved_bytes, ws = ctx.train_sizes(shape, T)
    ctx.ensure_workspace(ws)
    saved = torch.empty(saved_bytes, dtype=torch.uint8, device="cuda")
    Y, db1, db2 = torch.empty_like(X), torch.full((m,), 7.0, device="cuda").bfloat16(), torch.full((d,), 7.0, device="cuda").bfloat16()
    for _ in range(2):
        ctx.train_forward(shape, W1, None, W2, None, X, Y, saved=saved)
        ctx.train_backward(shape, W1, None, W2, X, saved, dY, db1=db1, db2=db2)
    ctx.poll()
    want = dY.double().sum(0)
    assert float((db2.double() - want).norm() / want.norm()) <= NORM_TOL["bf16"]
    some = torch.arange(0, m, 997, device="cuda")
    z = (X.double() @ W1[:, some].double()).requires_grad_()
    torch.nn.functional.gelu(z, approximate="tanh").backward(dY.double() @ W2[some].double().t())
    want = z.grad.sum(0)
    assert float((db1[some].double() - want).norm() / want.norm()) <= NORM_TOL["bf16"]


def ffn64_on_the_device(D, act):
    """ffn64() with torch, for layers that would take the host long."""
    z = D["X"] @ D["W1"] + (0 if D["b1"] is None else D["b1"])
    if act == "swiglu":
        s = torch.sigmoid(z)
        a, slope = z * s, s * (1 + z * (1 - s))
    elif act == "gelu_erf":
        phi = torch.special.ndtr(z)
        a, slope = z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    else:
        c, k = math.sqrt(2 / math.pi), 0.044715
        t = torch.tanh(c * (z + k * z ** 3))
        a, slope = 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * k * z * z)
    u = None if D["W1u"] is None else D["X"] @ D["W1u"]
    h = a if u is None else a * u
    dh = D["dY"] @ D["W2"].t()
    dz = dh * slope if u is None else dh * slope * u
    r = {"Y": h @ D["W2"] + (0 if D["b2"] is None else D["b2"]), "dX": dz @ D["W1"].t(), "dW1": D["X"].t() @ dz,
         "dW2": h.t() @ D["dY"], "db2": D["dY"].sum(0)}
    if u is not None:
        r["dX"] += (dh * a) @ D["W1u"].t()
        r["dW1u"] = D["X"].t() @ (dh * a)
    else:
        r["db1"] = dz.sum(0)
    return r


def draw_on_the_device(act, dtype, d, m, T, seed=0):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + d + 7 * m + 13 * T)
    new = lambda s, *shape: (torch.randn(*shape, generator=g, device="cuda") * s).to(DT[dtype])  # noqa: E731
    gated, w = act == "swiglu", 1.3 / math.sqrt(d)
    return {"X": new(1.0, T, d), "W1": new(w, d, m), "W1u": new(w, d, m) if gated else None, "b1": None if gated else new(0.2, m),
            "W2": new(1 / math.sqrt(m), m, d), "b2": new(0.2, d), "dY": new(0.01, T, d)}


def check_on_the_device(got, D, act, dtype, tol=None):
    ref = ffn64_on_the_device({k: None if v is None else v.double() for k, v in D.items()}, act)
    tol = NORM_TOL[dtype] if tol is None else tol
    for k, v in got.items():
        off = v.cuda().double() - ref[k]
        err, big = float(off.norm() / ref[k].norm()), float(off.abs().max() / ref[k].abs().max())
        assert err <= tol and big <= 8 * tol, f"{k}: {err:.2e} of the norm (<= {tol}), {big:.2e} of the largest element"


@pytest.mark.parametrize("dtype,act,d,m,T", [
    ("f32", "gelu_erf", 1026, 4096, 128), ("f32", "swiglu", 1001, 4096, 64),                  # dW1, dW1u whole pieces, dW2 not
    ("bf16", "swiglu", 4416, 517, 71), ("bf16", "gelu_erf", 5120, 20479, 300)])               # dX whole pieces, dW1, dW1u not
def test_gradients_that_leave_in_both_ways(ctx, dtype, act, d, m, T):
    """Gradients whose rows start on 16 bytes leave through TMA stores, others word by word, both through the same staging
    buffers.  Here pairs of CTAs go from a tile of the one kind straight to a short one of the other (59, 54, 24 and 40 times)."""
    D = draw_on_the_device(act, dtype, d, m, T)
    first = run(ctx, D, act, dtype)
    check_on_the_device(first, D, act, dtype)
    for _ in range(4):
        again = run(ctx, D, act, dtype)
        for k in first:
            assert torch.equal(again[k], first[k]), k


@pytest.mark.parametrize("act,d,m,T", [("swiglu", 1024, 2752, 1024), ("gelu_erf", 256, 1024, 128), ("gelu_tanh", 640, 4096, 2048)])
def test_long_fp32_sums(ctx, act, d, m, T):
    """The tensor cores cut their running sums (3e-8 of the sum to an MMA), so a sum leaves them every eighth MMA: 2.4e-7 of
    it at most, however long.  Two products in a row and the roundings of 2^-24 in between: 5e-7 of the norm."""
    D = draw_on_the_device(act, "f32", d, m, T)
    check_on_the_device(run(ctx, D, act, "f32"), D, act, "f32", tol=5e-7)


@pytest.mark.parametrize("act", ["swiglu", "gelu_erf", "gelu_tanh"])
def test_neurons_that_are_mostly_negative(ctx, act):
    """fp32, pre-activations around -4, neuron by neuron (whole-tensor norms hide the tail).  The value and the slope fall off
    like exp(-z^2 / 2): an error of Z counts |z| + 1 / |z| times, a rounded argument of the exponential z^2 2^-24 (the tanh
    form: three times that).  Down to z = -6 that is 4e-6 and up to 5e-6; with the products' 1e-6: the library's 1e-5."""
    D = draw_on_the_device(act, "f32", 256, 512, 200)
    D["W1"] *= 0.5 / 1.3
    D["X"][:, 0], D["W1"][0] = 1.0, -4.0
    got = {k: v.cuda().double() for k, v in run(ctx, D, act, "f32").items()}
    ref = ffn64_on_the_device({k: None if v is None else v.double() for k, v in D.items()}, act)
    for k, axis in (("dW1", 0), ("dW1u", 0), ("dW2", 1)):
        if k in got:
            off = (got[k] - ref[k]).norm(dim=axis) / ref[k].norm(dim=axis)
            assert float(off.max()) <= 1e-5, f"{k}: a neuron is {float(off.max()):.2e} off"
    if "db1" in got:      # (a sum that may cancel: held against the norm of its terms, which is a 16th of its neuron's in X^T dZ)
        off = (got["db1"] - ref["db1"]).abs() / (ref["dW1"].norm(dim=0) / 16)
        assert float(off.max()) <= 1e-5, f"db1: a neuron is {float(off.max()):.2e} off"


def test_directional_differences(ctx):
    """<gradient, direction> against central differences of the loss sum(Y * dY), fp32.  The direction is the
    gradient's own, scaled to a step of 1 % of the tensor: third-order terms are 1e-4 relative, the rounding of the
    loss (1e-5 of its terms) less than 1e-3 of a difference this large."""
    for act in ("swiglu", "gelu_erf", "gelu_tanh"):
        L = draw(act, "f32", 48, 96, 40, seed=5)
        got = run(ctx, L, act, "f32")
        weigh = L["dY"].double()
        for k in ("X", "W1", "W1u", "b1", "W2", "b2"):
            if L[k] is None:
                continue
            g = got["d" + k].double()
            step = 0.01 * L[k].double().norm() / g.norm()
            loss = []
            for sign in (1, -1):
                M = dict(L)
                M[k] = (L[k].double() + sign * step * g).float()
                loss.append(float((run(ctx, M, act, "f32", keep=False)["Y"].double() * weigh).sum()))
            slope = (loss[0] - loss[1]) / (2 * float(step))
            want = float((g * g).sum())
            assert abs(slope - want) <= 5e-3 * want, (act, k, slope, want)


def test_refusals(ctx):
    import paper_2401_04044_b200 as ff
    L = {k: None if v is None else v.cuda() for k, v in draw("swiglu", "bf16", 64, 96, 10).items()}
    shape = ff.make_shape(64, 96, "swiglu", torch.bfloat16)
    saved_bytes, ws = ctx.train_sizes(shape, 10)
    ctx.ensure_workspace(ws)
    saved = torch.empty(saved_bytes, dtype=torch.uint8, device="cuda")
    Y, dW1 = torch.empty_like(L["X"]), torch.empty_like(L["W1"])

    def fwd(**k):
        a = {**L, "Y": Y, "saved": saved, "shape": shape, **k}
        ctx.train_forward(a["shape"], a["W1"], a["b1"], a["W2"], a["b2"], a["X"], a["Y"], saved=a["saved"], W1u=a["W1u"])

    def bwd(**k):
        a = {**L, "saved": saved, "g": {"dW1": dW1}, **k}
        ctx.train_backward(shape, a["W1"], a["b1"], a["W2"], a["X"], a["saved"], a["dY"], W1u=a["W1u"], **a["g"])

    before = ctx.launch_count()
    bias = torch.zeros(96, dtype=torch.bfloat16, device="cuda")
    wide = torch.zeros(10, 128, dtype=torch.bfloat16, device="cuda")
    odd = torch.empty(10 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    for call, code in [
        (lambda: fwd(W1u=None), 1), (lambda: fwd(b1=bias), 1), (lambda: fwd(X=L["X"].float()), 4),
        (lambda: fwd(X=wide[:, :64]), 2), (lambda: fwd(X=L["X"].cpu()), 1), (lambda: fwd(W1=L["W1"].t()), 2),
        (lambda: fwd(X=L["X"][:0], Y=Y[:0]), 2), (lambda: fwd(saved=saved[:-1]), 5), (lambda: fwd(saved=saved[16:]), 3),
        (lambda: fwd(X=odd[1:641].view(10, 64)), 3), (lambda: fwd(Y=odd[1:641].view(10, 64)), 3),
        (lambda: bwd(g={}), 1), (lambda: bwd(saved=None), 1), (lambda: bwd(g={"db1": bias}), 1),
        (lambda: bwd(g={"dW1": dW1.float()}), 4), (lambda: bwd(g={"dW1": dW1[:-1]}), 2), (lambda: bwd(dY=L["dY"][:5]), 2),
        (lambda: ctx.train_sizes(shape, 0), 2), (lambda: ctx.train_sizes(ff.make_shape(60, 96, "swiglu", torch.bfloat16), 4), 2),
    ]:
        with pytest.raises(ff.FFSplitError) as e:
            call()
        assert e.value.code == code
    assert ctx.launch_count() == before
    small = ff.Context(0)
    small.ensure_workspace(1 << 16)
    with pytest.raises(ff.FFSplitError) as e:
        small.train_forward(shape, L["W1"], None, L["W2"], None, L["X"], Y, W1u=L["W1u"])
    assert e.value.code == 5
    small.close()


def test_scoring_after_training_prepares_its_weights_again(ctx):
    """Scoring keeps transposed weights in the workspace between the batches of one accumulation; a training call in
    between writes over them."""
    import paper_2401_04044_b200 as ff
    L = {k: None if v is None else v.cuda() for k, v in draw("gelu_erf", "bf16", 64, 256, 200).items()}
    shape = ff.make_shape(64, 256, "gelu_erf", torch.bfloat16)
    ctx.ensure_workspace(max(ctx.workspace_size(shape, 0, 200, 0, 0), ctx.train_sizes(shape, 200)[1]))
    out = []
    for train in (False, True):
        e = torch.empty(256, device="cuda")
        ctx.score(shape, L["W1"], L["b1"], L["W2"], L["X"], e)
        if train:
            Y = torch.empty_like(L["X"])
            ctx.train_forward(shape, L["W1"], L["b1"], L["W2"], L["b2"], L["X"], Y)
        ctx.score(shape, L["W1"], L["b1"], L["W2"], L["X"], e, accumulate=True)
        ctx.poll()
        out.append(e.clone())
    assert torch.equal(out[0], out[1])


# ------------------------------------------------------------------------------------------------ norm and clipping
def views(sizes, kinds, seed, scale=1.0, gap=0):
    """Gradients as views of one flat buffer to a type, `gap` elements apart (odd ones start off 16 bytes)."""
    g = torch.Generator().manual_seed(seed)
    flat = {k: torch.randn(max(1, sum(n + gap for n, t in zip(sizes, kinds) if t == k)), generator=g).mul_(scale).to(DT[k]).cuda()
            for k in set(kinds)}
    at = {k: 0 for k in flat}
    out = []
    for n, k in zip(sizes, kinds):
        out.append(flat[k][at[k]:at[k] + n])
        at[k] += n + gap
    return out


def norm64(ts):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in ts))


def clip_both(ctx, grads, max_norm, out=None):
    ctx.ensure_workspace(ctx.grad_workspace_size(len(grads)))
    norm = torch.empty(1, device="cuda")
    lst = ctx.grad_list(grads, out)
    ctx.clip_grads(lst, max_norm, norm)
    ctx.poll()
    return float(norm)


CLIP_SIZES = [
    [1], [0], [7, 0, 1], [8, 16, 24], [16384], [16385, 16383], [100003, 3, 70000, 0, 1], list(range(1, 300)), [5] * 1100 + [40000],
]


@pytest.mark.parametrize("sizes", CLIP_SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("kind", ["bf16", "f32", "mixed"])
@pytest.mark.parametrize("gap", [0, 3])
def test_norm_and_clipping(ctx, sizes, kind, gap):
    kinds = [kind if kind != "mixed" else ("f32", "bf16")[i % 2] for i in range(len(sizes))]
    grads = views(sizes, kinds, seed=len(sizes), gap=gap)
    keep = [g.clone() for g in grads]
    want = norm64(keep)
    # squares in runs of 8 and a rounding to fp32 at the end: 2^-24 times a few
    ctx.ensure_workspace(ctx.grad_workspace_size(len(grads)))
    norm = torch.empty(1, device="cuda")
    ctx.grad_norm(ctx.grad_list(grads), norm)
    ctx.poll()
    assert abs(float(norm) - want) <= 5e-7 * want
    # elsewhere first, with the outputs at another offset from 16 bytes; then in place
    outs = [torch.full((g.numel() + 3,), -7.0, dtype=g.dtype, device="cuda") for g in grads]
    elsewhere = [o[1:1 + g.numel()] for o, g in zip(outs, grads)]
    for max_norm in (0.37 * want + 1e-3, 2 * want + 1.0, 0.0, float("inf")):
        factor = min(1.0, max_norm / (want + 1e-6))
        for out in (elsewhere, grads):
            got_norm = clip_both(ctx, grads, max_norm, None if out is grads else out)
            assert abs(got_norm - want) <= 5e-7 * want
            for o, k in zip(out, keep):
                r = k.double() * factor
                # one rounding to the type of a product whose factor is off by a few 2^-24
                tol = (2.0 ** -8 if k.dtype == torch.bfloat16 else 1e-6) * r.abs()
                assert ((o.double() - r).abs() <= tol).all()
                if factor == 1.0:
                    assert torch.equal(o, k)
        for o, g in zip(outs, keep):
            assert o[0] == -7 and (o[1 + g.numel():] == -7).all()
        for g, k in zip(grads, keep):
            g.copy_(k)


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e19, 1e30])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_norm_outside_the_range_of_fp32_squares(ctx, scale, kind):
    grads = views([1000, 3, 70001], [kind] * 3, seed=2, scale=scale)
    norm = torch.empty(1, device="cuda")
    ctx.ensure_workspace(ctx.grad_workspace_size(3))
    ctx.grad_norm(ctx.grad_list(grads), norm)
    ctx.poll()
    want = norm64(grads)
    assert abs(float(norm) - want) <= 5e-7 * want


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-3, 1e-38, 1e-40])
def test_norm_of_mostly_zeros(ctx, kind, scale):
    """Zeros of both signs everywhere but in a few places, whose values may be subnormal and have squares that are not."""
    grads = [torch.zeros(n, dtype=DT[kind], device="cuda") for n in (100_000, 7, 40_001)]
    grads[0][::2] *= -1
    for g, places in zip(grads, ((3, 4096, 77_777), (6,), (0, 40_000))):
        for i in places:
            g[i] = (i % 5 + 1) * scale
    norm = torch.empty(1, device="cuda")
    ctx.ensure_workspace(ctx.grad_workspace_size(3))
    ctx.grad_norm(ctx.grad_list(grads), norm)
    ctx.poll()
    want = norm64(grads)
    assert want > 0 and abs(float(norm) - want) <= 5e-7 * want + 2.0 ** -150     # (half a step of the subnormal numbers)
    for g in grads:
        g.zero_()
    ctx.grad_norm(ctx.grad_list(grads), norm)
    ctx.poll()
    assert float(norm) == 0.0


def test_clipping_an_empty_list(ctx):
    assert clip_both(ctx, [], 1.0) == 0.0


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_non_finite_norm_is_reported_and_changes_nothing(ctx, bad):
    import paper_2401_04044_b200 as ff
    grads = views([500, 33], ["f32", "bf16"], seed=4)
    grads[1][7] = bad
    keep = [g.clone() for g in grads]
    norm = torch.empty(1, device="cuda")
    ctx.ensure_workspace(ctx.grad_workspace_size(2))
    ctx.clip_grads(ctx.grad_list(grads), 0.1, norm)
    with pytest.raises(ff.FFSplitError) as e:
        ctx.poll()
    assert e.value.code == 6
    assert not math.isfinite(float(norm))
    for g, k in zip(grads, keep):
        assert torch.equal(g.view(torch.int32 if g.dtype == torch.float32 else torch.int16),
                           k.view(torch.int32 if k.dtype == torch.float32 else torch.int16))
    ctx.poll()


def test_clipping_refusals(ctx):
    import paper_2401_04044_b200 as ff
    g = torch.ones(100, device="cuda")
    norm = torch.empty(1, device="cuda")
    ctx.ensure_workspace(ctx.grad_workspace_size(1))
    before = ctx.launch_count()
    for call, code in [
        (lambda: ctx.grad_list([g.half()]), 4), (lambda: ctx.grad_list([g], [g.bfloat16()]), 4),
        (lambda: ctx.grad_list([g], [g[:50]]), 2), (lambda: ctx.grad_list([g[::2]]), 2), (lambda: ctx.grad_list([g.cpu()]), 1),
        (lambda: ctx.grad_list([g], []), 2), (lambda: ctx.clip_grads(ctx.grad_list([g]), -1.0, norm), 1),
        (lambda: ctx.clip_grads(ctx.grad_list([g]), float("nan"), norm), 1),
        (lambda: ctx.clip_grads(ctx.grad_list([g]), 1.0, norm.double()), 2),
    ]:
        with pytest.raises(ff.FFSplitError) as e:
            call()
        assert e.value.code == code
    assert ctx.launch_count() == before
    small = ff.Context(0)
    small.ensure_workspace(1 << 16)
    with pytest.raises(ff.FFSplitError) as e:
        small.grad_norm(small.grad_list([g]), norm)
    assert e.value.code == 5
    small.close()


# ------------------------------------------------------------------------------------------------ through PyTorch
@pytest.mark.parametrize("act", ["swiglu", "gelu_erf"])
def test_autograd_function_matches_the_calls(ctx, act):
    from paper_2401_04044_b200 import make_shape
    from paper_2401_04044_b200.train import ffn
    L = draw(act, "bf16", 72, 200, 90)
    want = run(ctx, L, act, "bf16")
    D = {k: None if v is None else v.cuda().requires_grad_(k != "dY") for k, v in L.items()}
    Y = ffn(ctx, make_shape(72, 200, act, torch.bfloat16), D["X"], D["W1"], D["W2"], D["b1"], D["b2"], D["W1u"])
    Y.backward(D["dY"])
    assert torch.equal(Y.detach().cpu(), want["Y"])
    for k, t in D.items():
        if t is not None and k != "dY":
            assert torch.equal(t.grad.cpu(), want["d" + k]), k
    # frozen weights: only what is needed is computed
    X = D["X"].detach().requires_grad_()
    Y = ffn(ctx, make_shape(72, 200, act, torch.bfloat16), X, *(D[k] if D[k] is None else D[k].detach() for k in ("W1", "W2", "b1", "b2", "W1u")))
    Y.backward(D["dY"])
    assert torch.equal(X.grad.cpu(), want["dX"])


def test_autograd_function_keeps_nothing_without_grad_and_has_no_second_derivative(ctx):
    from paper_2401_04044_b200 import make_shape
    from paper_2401_04044_b200.train import ffn
    D = {k: None if v is None else v.cuda().requires_grad_(k == "X") for k, v in draw("swiglu", "bf16", 256, 512, 2000).items()}
    shape = make_shape(256, 512, "swiglu", torch.bfloat16)
    call = lambda: ffn(ctx, shape, D["X"], D["W1"], D["W2"], W1u=D["W1u"])  # noqa: E731
    want = call()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.max_memory_allocated()
    with torch.no_grad():
        Y = call()
    assert torch.equal(Y, want.detach())
    assert torch.cuda.max_memory_allocated() - before < ctx.train_sizes(shape, 2000)[0]
    (g,) = torch.autograd.grad(want, D["X"], D["dY"].requires_grad_(), create_graph=True)
    with pytest.raises(RuntimeError):
        g.float().sum().backward()


@pytest.mark.parametrize("d,rows", [(33, (7, 12)), (35, (1, 2)), (34, (5, 6))])
def test_autograd_function_takes_gradients_that_start_anywhere(ctx, d, rows):
    """Behind torch.cat, a layer's gradient is a piece of a larger one; behind a sum it is one number, expanded."""
    from paper_2401_04044_b200 import make_shape
    from paper_2401_04044_b200.train import ffn
    L = draw("gelu_erf", "f32", d, 40, sum(rows))
    shape, D = make_shape(d, 40, "gelu_erf", torch.float32), {k: None if v is None else v.cuda() for k, v in L.items()}
    layer = lambda X: ffn(ctx, shape, X, D["W1"], D["W2"], D["b1"], D["b2"])  # noqa: E731
    X = D["X"].clone().requires_grad_()
    pieces = [x.clone() for x in X.split(rows)]      # (as inputs, the pieces have to be aligned)
    torch.cat([layer(x) for x in pieces]).backward(D["dY"])
    check({"dX": X.grad.cpu()}, L, "gelu_erf", "f32")
    X = D["X"].clone().requires_grad_()
    layer(X).sum().backward()
    check({"dX": X.grad.cpu()}, {**L, "dY": torch.ones_like(L["dY"])}, "gelu_erf", "f32")


@pytest.mark.parametrize("dtype,act,T", [("bf16", "swiglu", 90), ("bf16", "gelu_erf", 700), ("f32", "gelu_tanh", 33)])
def test_a_captured_pass_reads_its_inputs_anew(ctx, dtype, act, T):
    """Forward, backward and clipping as one CUDA graph, replayed on other inputs than it was captured with."""
    import paper_2401_04044_b200 as ff
    d, m = 72, 203
    first, other = ({k: None if v is None else v.cuda() for k, v in draw(act, dtype, d, m, T).items()} for _ in range(2))
    for k in other:
        if other[k] is not None:
            other[k] = (other[k].float() * -0.75).to(DT[dtype])
    shape = ff.make_shape(d, m, act, DT[dtype])
    saved_bytes, ws = ctx.train_sizes(shape, T)
    ctx.ensure_workspace(max(ws, ctx.grad_workspace_size(3)))
    saved, Y, norm = torch.empty(saved_bytes, dtype=torch.uint8, device="cuda"), torch.empty_like(first["X"]), torch.zeros(1, device="cuda")
    g = {"d" + k: torch.empty_like(first[k]) for k in ("X", "W1", "W1u", "b1", "W2", "b2")
         if first[k] is not None and not (act == "swiglu" and k == "b1")}
    grads = ctx.grad_list([g["dX"], g["dW1"], g["dW2"]])

    def step():
        ctx.train_forward(shape, first["W1"], first["b1"], first["W2"], first["b2"], first["X"], Y, saved=saved, W1u=first["W1u"])
        ctx.train_backward(shape, first["W1"], None, first["W2"], first["X"], saved, first["dY"], W1u=first["W1u"], **g)
        ctx.clip_grads(grads, 0.5, norm)

    step()      # sets the kernels' attributes, which a capture may not
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k, v in first.items():
        if v is not None:
            v.copy_(other[k])
    step()
    want = {k: v.clone() for k, v in {**g, "Y": Y, "norm": norm}.items()}
    for v in (*g.values(), Y, norm):
        v.zero_()
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(v, want[k]) for k, v in {**g, "Y": Y, "norm": norm}.items())


def test_saved_has_to_lie_on_the_device(ctx):
    import paper_2401_04044_b200 as ff
    L = {k: None if v is None else v.cuda() for k, v in draw("swiglu", "bf16", 64, 96, 10).items()}
    shape = ff.make_shape(64, 96, "swiglu", torch.bfloat16)
    saved_bytes, ws = ctx.train_sizes(shape, 10)
    ctx.ensure_workspace(ws)
    before = ctx.launch_count()
    host, gaps = torch.empty(saved_bytes, dtype=torch.uint8), torch.empty(2 * saved_bytes, dtype=torch.uint8, device="cuda")[::2]
    for saved in (host, gaps):
        for call in (lambda: ctx.train_forward(shape, L["W1"], None, L["W2"], None, L["X"], torch.empty_like(L["X"]), saved=saved, W1u=L["W1u"]),
                     lambda: ctx.train_backward(shape, L["W1"], None, L["W2"], L["X"], saved, L["dY"], dX=torch.empty_like(L["X"]), W1u=L["W1u"])):
            with pytest.raises(ff.FFSplitError) as e:
                call()
            assert e.value.code == 1
    assert ctx.launch_count() == before


def test_calls_from_a_thread_that_has_used_no_gpu(ctx):
    """Autograd runs backward passes on threads of its own, on which no CUDA context is current yet."""
    import threading
    L = draw("swiglu", "bf16", 72, 200, 90)
    want, got = run(ctx, L, "swiglu", "bf16"), {}
    t = threading.Thread(target=lambda: got.update(run(ctx, L, "swiglu", "bf16")))
    t.start()
    t.join()
    assert got and all(torch.equal(got[k], want[k]) for k in want)


def test_clip_grad_norm_in_place(ctx):
    from paper_2401_04044_b200.train import clip_grad_norm_
    ps = [torch.nn.Parameter(torch.zeros(n, dtype=t, device="cuda")) for n, t in ((1000, torch.bfloat16), (33, torch.float32), (5, torch.float32))]
    for p in ps[:2]:
        p.grad = torch.randn_like(p)
    want = norm64([p.grad for p in ps[:2]])
    norm = clip_grad_norm_(ctx, ps, 0.5)
    ctx.poll()
    assert abs(float(norm) - want) <= 5e-7 * want
    assert abs(norm64([p.grad for p in ps[:2]]) - 0.5) < 2e-3


def test_clip_grad_norm_of_one_tensor_and_of_a_tied_parameter(ctx):
    from paper_2401_04044_b200.train import clip_grad_norm_
    p = torch.nn.Parameter(torch.zeros(40, 25, device="cuda"))
    g = torch.randn(40, 25, device="cuda")
    want = norm64([g])
    for parameters in (p, [p, p]):
        p.grad = g.clone()
        norm = clip_grad_norm_(ctx, parameters, 0.5)
        ctx.poll()
        assert abs(float(norm) - want) <= 5e-7 * want
        assert abs(norm64([p.grad]) - 0.5) < 1e-5


@pytest.mark.parametrize("act", ["swiglu", "gelu_tanh"])
def test_finetuning_recovers_a_rounded_layer(ctx, act):
    from paper_2401_04044_b200.train import finetune
    losses, shape, W = finetune(ctx, 128, 320, act, tokens=256, steps=25)
    assert shape.m == 320 and all(math.isfinite(v) for v in losses)
    assert sum(losses[-5:]) < 0.8 * sum(losses[:5])


# ------------------------------------------------------------------------------------------------ the shared workspace
SLEEP = 50_000_000      # cycles: some 30 ms of a stream that is busy


def test_a_new_workspace_is_clear_for_calls_on_any_stream(ctx):
    """The control block of a workspace full of other data is cleared before calls on a side stream read its tickets, though
    the default stream, on which the library clears it, is busy."""
    import paper_2401_04044_b200 as ff
    d, m, T = 72, 200, 1600      # (db2's rows are cut: its blocks take tickets)
    L = draw("gelu_erf", "bf16", d, m, T)
    want = run(ctx, L, "gelu_erf", "bf16")
    D = {k: None if v is None else v.cuda() for k, v in L.items()}
    shape = ff.make_shape(d, m, "gelu_erf", torch.bfloat16)
    saved_bytes, ws = ctx.train_sizes(shape, T)
    saved, Y = torch.empty(saved_bytes, dtype=torch.uint8, device="cuda"), torch.empty_like(D["X"])
    g = {"d" + k: torch.zeros_like(D[k]) for k in ("X", "W1", "b1", "W2", "b2")}
    memory, side, fresh = torch.full((ws,), 0xFF, dtype=torch.uint8, device="cuda"), torch.cuda.Stream(), ff.Context(0)
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    with torch.cuda.stream(side):
        fresh.set_workspace(memory)
        fresh.train_forward(shape, D["W1"], D["b1"], D["W2"], D["b2"], D["X"], Y, saved=saved)
        fresh.train_backward(shape, D["W1"], None, D["W2"], D["X"], saved, D["dY"], **g)
        fresh.poll()
    assert all(torch.equal(v.cpu(), want[k]) for k, v in g.items())
    fresh.close()


def test_pytorch_calls_grow_the_workspace_on_a_side_stream(ctx):
    """A fresh context used on a side stream only, nothing synchronised in between; the workspace takes memory that work queued
    on that stream has yet to read."""
    import paper_2401_04044_b200 as ff
    from paper_2401_04044_b200.train import clip_grad_norm_, ffn
    d, m, T = 72, 200, 1600
    L = draw("gelu_erf", "bf16", d, m, T)
    want = run(ctx, L, "gelu_erf", "bf16")
    shape = ff.make_shape(d, m, "gelu_erf", torch.bfloat16)
    D = {k: None if v is None else v.cuda().requires_grad_(k != "dY") for k, v in L.items()}
    side, fresh = torch.cuda.Stream(), ff.Context(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        memory = torch.full((ctx.train_sizes(shape, T)[1],), 0xFF, dtype=torch.uint8, device="cuda")
        torch.cuda._sleep(SLEEP)
        seen = memory[:1 << 16].clone()
        del memory
        Y = ffn(fresh, shape, D["X"], D["W1"], D["W2"], D["b1"], D["b2"])
        Y.backward(D["dY"])
        grads = {k: v.grad.clone() for k, v in D.items() if v is not None and k != "dY"}
        norm = clip_grad_norm_(fresh, [v for k, v in D.items() if v is not None and k != "dY"], 0.5)
        fresh.poll()
    assert (seen == 0xFF).all()
    assert torch.equal(Y.detach().cpu(), want["Y"]) and all(torch.equal(v.cpu(), want["d" + k]) for k, v in grads.items())
    assert abs(float(norm) - norm64(list(grads.values()))) <= 5e-7 * float(norm)
    fresh.close()


def test_a_non_finite_norm_is_reported_after_the_workspace_has_grown(ctx):
    import paper_2401_04044_b200 as ff
    from paper_2401_04044_b200.train import clip_grad_norm_, ffn
    D = {k: None if v is None else v.cuda() for k, v in draw("swiglu", "bf16", 64, 96, 50).items()}
    p, fresh = torch.nn.Parameter(torch.zeros(100, device="cuda")), ff.Context(0)
    p.grad = torch.full_like(p, float("inf"))
    clip_grad_norm_(fresh, p, 1.0)
    ffn(fresh, ff.make_shape(64, 96, "swiglu", torch.bfloat16), D["X"], D["W1"], D["W2"], W1u=D["W1u"])
    with pytest.raises(ff.FFSplitError) as e:
        fresh.poll()
    assert e.value.code == 6
    fresh.poll()
    fresh.close()


def test_a_captured_pass_outlives_its_workspace(ctx):
    """After the capture a larger call replaces the workspace and other tensors take what memory is free; replays neither read
    those nor write to them."""
    import paper_2401_04044_b200 as ff
    D = {k: None if v is None else v.cuda() for k, v in draw("gelu_erf", "f32", 130, 257, 300).items()}
    shape, fresh = ff.make_shape(130, 257, "gelu_erf", torch.float32), ff.Context(0)
    saved_bytes, ws = fresh.train_sizes(shape, 300)
    fresh.ensure_workspace(ws)
    saved, Y = torch.empty(saved_bytes, dtype=torch.uint8, device="cuda"), torch.empty_like(D["X"])
    g = {"d" + k: torch.empty_like(D[k]) for k in ("X", "W1", "b1", "W2", "b2")}

    def step():
        fresh.train_forward(shape, D["W1"], D["b1"], D["W2"], D["b2"], D["X"], Y, saved=saved)
        fresh.train_backward(shape, D["W1"], None, D["W2"], D["X"], saved, D["dY"], **g)

    step()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in {**g, "Y": Y}.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    fresh.ensure_workspace(8 * ws)
    others = [torch.full((ws,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]
    for v in (*g.values(), Y):
        v.zero_()
    graph.replay()
    fresh.poll()
    assert all(torch.equal(v, want[k]) for k, v in {**g, "Y": Y}.items())
    assert all((o == 0x5A).all() for o in others)
    with pytest.raises(ff.FFSplitError) as e:
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            step()
            fresh.ensure_workspace(16 * ws)
    assert e.value.code == 1
    torch.cuda.synchronize()
    fresh.close()
