"""The training operators, as they are measured: the feed-forward block's forward, its forward and backward as a
training step runs them, and the global gradient norm with clipping.

`run` computes a case in its plain form (elementary torch operations in 32 bits, rounded once at the end), or with
`own` through the library's entry points; `exact` is the same result from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------- the cases
def _ffn(name, kind, d, m, T, act, dtype):
    return {"name": name, "kind": kind, "d": d, "m": m, "T": T, "act": act, "dtype": dtype}


def _clip(name, sizes, dtype, norm, seed_sizes=0):
    return {"name": name, "kind": "clip", "sizes": sizes, "dtype": dtype, "norm": norm, "seed_sizes": seed_sizes}


def listed():
    return [
        # one token through a 4096 x 11008 gated layer (a generation step while the weights are still being trained)
        _ffn("forward gated T1", "forward", 4096, 11008, 1, "swiglu", "bf16"),
        # a small gated layer and few tokens: what counts is the latency of the calls
        _ffn("forward gated small", "forward", 256, 1024, 64, "swiglu", "bf16"),
        # validation loss over long batches: forward alone, nothing kept for a backward pass
        _ffn("forward gated T8192", "forward", 4096, 11008, 8192, "swiglu", "bf16"),
        # fine-tuning a gated layer of the same shape on one 2048-token sequence
        _ffn("train gated T2048", "train", 4096, 11008, 2048, "swiglu", "bf16"),
        # fine-tuning a 5120 x 20480 GELU layer with biases: the largest step
        _ffn("train gelu T4096", "train", 5120, 20480, 4096, "gelu_erf", "bf16"),
        # a 1024 x 4096 layer (tanh form) on a ragged batch
        _ffn("train gelu_tanh T1000", "train", 1024, 4096, 1000, "gelu_tanh", "bf16"),
        # widths that fill no tile: neurons left over after others were removed, and an odd token count
        _ffn("train gated ragged", "train", 1000, 2731, 777, "swiglu", "bf16"),
        # 32-bit training: the smallest layer, and a gated one in the middle of the range
        _ffn("train gelu f32 small", "train", 256, 1024, 128, "gelu_erf", "f32"),
        _ffn("train gated f32", "train", 1024, 2752, 1024, "swiglu", "f32"),
        # gradients of four 4096 x 11008 gated layers, over the limit
        _clip("clip 12 matrices bf16", "gated4096x11008x4", "bf16", 7.5),
        # many small tensors of both types, odd sizes: biases, norms and adapters of a whole model, over the limit
        _clip("clip 400 small mixed", "random400x1200000", "mixed", 3.0, 11),
        # 32-bit gradients of a 24-layer 1024 x 4096 stack with biases, under the limit
        _clip("clip 24 layers f32", "gelu1024x4096x24", "f32", 0.4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["forward", "train", "train", "clip"])
    if kind == "clip":
        n = _log_int(rng, 1, 600)
        total = max(4 * n, _log_int(rng, 1000, 400_000_000))
        return {"kind": "clip", "sizes": "random%dx%d" % (n, total), "dtype": rng.choice(["bf16", "f32", "mixed"]),
                "norm": round(math.exp(rng.uniform(math.log(0.1), math.log(30.0))), 3), "seed_sizes": rng.randrange(1, 1 << 30)}
    dtype = rng.choice(["bf16", "bf16", "f32"])
    act = rng.choice(["swiglu", "swiglu", "gelu_erf", "gelu_tanh"])
    big = 1.0 if dtype == "bf16" else 0.4     # 32-bit layers stay smaller
    d = _log_int(rng, 64, int(5120 * big))
    if dtype == "bf16":
        d = d // 8 * 8                        # rows of 16 bytes, as everywhere in the library
    m = _log_int(rng, 64, int(20480 * big))
    T = _log_int(rng, 1, 8192)
    limit = 0.9 * max(_flops(c) for c in listed() if c["kind"] == "train")
    case = {"kind": kind, "d": d, "m": m, "T": T, "act": act, "dtype": dtype}
    case["T"] = max(1, min(T, int(T * limit / _flops(case))))
    return case


def _flops(case):
    products = 3 if case["act"] == "swiglu" else 2
    return 2.0 * products * case["T"] * case["d"] * case["m"] * (3 if case["kind"] == "train" else 1)


def _sizes(case):
    """Element counts of a clip case's tensors, from its text."""
    s = case["sizes"]
    if s.startswith("gated"):
        d, m, layers = (int(v) for v in s[5:].split("x"))
        return [d * m] * (3 * layers)
    if s.startswith("gelu"):
        d, m, layers = (int(v) for v in s[4:].split("x"))
        return [d * m, m, m * d, d] * layers
    n, total = (int(v) for v in s[6:].split("x"))
    r = random.Random(case["seed_sizes"])
    share = [math.exp(r.gauss(0.0, 1.5)) for _ in range(n)]
    whole = sum(share)
    return [max(1, int(total * v / whole)) for v in share]


def _kinds(case, n):
    """The types of a clip case's n tensors."""
    if case["dtype"] != "mixed":
        return [DTYPES[case["dtype"]]] * n
    return [torch.float32 if i % 3 == 0 else torch.bfloat16 for i in range(n)]


def work(case):
    if case["kind"] == "clip":
        sizes = _sizes(case)
        held = sum(n * (4 if t is torch.float32 else 2) for n, t in zip(sizes, _kinds(case, len(sizes))))
        return {"bytes": 2.0 * held + 4, "flops": 3.0 * sum(sizes)}
    e = 2 if case["dtype"] == "bf16" else 4
    d, m, T, gated = case["d"], case["m"], case["T"], case["act"] == "swiglu"
    weights = (3 if gated else 2) * d * m + (0 if gated else m + d)
    times = 2 if case["kind"] == "train" else 1    # a training step also reads dY and writes dX and the weights' gradients
    return {"bytes": float(e * times * (2 * T * d + weights)), "flops": _flops(case)}


# ---------------------------------------------------------------------------------------------------- inputs
def _draw_ffn(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + case["d"] * 31 + case["m"] * 17 + case["T"])
    dt, d, m, T = DTYPES[case["dtype"]], case["d"], case["m"], case["T"]
    new = lambda scale, *shape: (torch.randn(*shape, generator=g, device="cuda") * scale).to(dt)  # noqa: E731
    gated = case["act"] == "swiglu"
    return {
        "X": new(1.0, T, d),                           # normalised activations
        "W1": new(0.02 if d >= 1024 else 0.06, d, m),
        "W1u": new(0.02 if d >= 1024 else 0.06, d, m) if gated else None,
        "b1": None if gated else new(0.1, m),
        "W2": new(0.02, m, d),
        "b2": None if gated else new(0.1, d),
        "dY": new(1e-3, T, d) if case["kind"] == "train" else None,   # the gradient of a mean loss
    }


def _draw_grads(case, seed):
    """The gradients as training programs hold them: one flat buffer to a type, tensor after tensor without gaps (so
    that most odd ones start off a 16-byte boundary).  -> {type name: flat buffer}, list of views in the tensors' order"""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 5)
    sizes = _sizes(case)
    kinds = _kinds(case, len(sizes))
    r = random.Random(case["seed_sizes"] + 1)
    scale = [math.exp(r.uniform(-3.0, 3.0)) for _ in sizes]             # layers differ in the size of their gradients
    norm = math.sqrt(sum(n * s * s for n, s in zip(sizes, scale)))
    flat = {}
    for name, t in DTYPES.items():
        mine = [i for i, k in enumerate(kinds) if k is t]
        if mine:
            factor = torch.repeat_interleave(torch.tensor([scale[i] * case["norm"] / norm for i in mine], device="cuda"),
                                             torch.tensor([sizes[i] for i in mine], device="cuda"))
            flat[name] = factor.mul_(torch.randn(factor.numel(), generator=g, device="cuda")).to(t)
    return flat, _views(case, flat)


def _views(case, flat):
    sizes = _sizes(case)
    kinds = _kinds(case, len(sizes))
    parts = {DTYPES[k]: iter(torch.split(v, [n for n, t in zip(sizes, kinds) if t is DTYPES[k]])) for k, v in flat.items()}
    return [next(parts[t]) for t in kinds]


_library = {}


def _context():
    """The library's context, one to a process."""
    if "ctx" not in _library:
        from paper_2401_04044_b200 import Context
        _library["ctx"] = Context(0)
    return _library["ctx"]


def prepare(case, seed):
    """The inputs; with `own` also what a program that uses the library keeps between calls: the context with its
    workspace, the buffers for results, and the list that names the gradients.  Nothing is computed from the inputs."""
    if case["kind"] == "clip":
        flat, grads = _draw_grads(case, seed)
        state = {"case": case, "flat": flat, "grads": grads, "max_norm": 1.0}
        if own:
            ctx = _context()
            state["out"] = {k: torch.empty_like(v) for k, v in flat.items()}
            state["norm"] = torch.empty(1, dtype=torch.float32, device="cuda")
            state["list"] = ctx.grad_list(grads, _views(case, state["out"]))
            ctx.ensure_workspace(ctx.grad_workspace_size(len(grads)))
        return state
    state = {"case": case, **_draw_ffn(case, seed)}
    if own:
        from paper_2401_04044_b200 import make_shape
        ctx = _context()
        state["shape"] = make_shape(case["d"], case["m"], case["act"], DTYPES[case["dtype"]])
        saved, workspace = ctx.train_sizes(state["shape"], case["T"])
        ctx.ensure_workspace(workspace)
        like = lambda t: None if t is None else torch.empty_like(t)  # noqa: E731
        state["Y"] = torch.empty_like(state["X"])
        if case["kind"] == "train":
            state["saved"] = torch.empty(saved, dtype=torch.uint8, device="cuda")
            state["grads"] = {"d" + k: like(state[k]) for k in ("X", "W1", "W1u", "b1", "W2", "b2")}
    return state


# ---------------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "clip":
        return _plain_clip(state["flat"], state["max_norm"])
    return _plain_ffn(state, kind == "train")


def _run_own(s):
    ctx, kind = _context(), s["case"]["kind"]
    if kind == "clip":
        ctx.clip_grads(s["list"], s["max_norm"], s["norm"])
        return {"norm": s["norm"], **s["out"]}
    if kind == "forward":
        ctx.train_forward(s["shape"], s["W1"], s["b1"], s["W2"], s["b2"], s["X"], s["Y"], W1u=s["W1u"])
        return {"Y": s["Y"]}
    ctx.train_forward(s["shape"], s["W1"], s["b1"], s["W2"], s["b2"], s["X"], s["Y"], saved=s["saved"], W1u=s["W1u"])
    ctx.train_backward(s["shape"], s["W1"], s["b1"], s["W2"], s["X"], s["saved"], s["dY"], W1u=s["W1u"], **s["grads"])
    return {"Y": s["Y"], **{k: v for k, v in s["grads"].items() if v is not None}}


def _plain_clip(flat, max_norm):
    wide = {k: v.float() for k, v in flat.items()}
    norm = torch.sqrt(sum((v * v).sum() for v in wide.values())).reshape(1)
    factor = torch.clamp(max_norm / (norm + 1e-6), max=1.0)
    return {"norm": norm, **{k: (v * factor).to(flat[k].dtype) for k, v in wide.items()}}


def _act_and_slope(z, act):
    """act(z) and its derivative in z's own type, from elementary operations."""
    if act == "swiglu":
        s = torch.sigmoid(z)
        return z * s, s * (1.0 + z * (1.0 - s))
    if act == "gelu_erf":
        phi = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    c, a = math.sqrt(2.0 / math.pi), 0.044715
    t = torch.tanh(c * (z + a * z * z * z))
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * (c * (1.0 + 3.0 * a * z * z))


def _plain_ffn(s, train):
    act, dt = s["case"]["act"], s["X"].dtype
    f = lambda t: None if t is None else t.float()  # noqa: E731
    X, W1, W1u, W2, b1, b2 = (f(s[k]) for k in ("X", "W1", "W1u", "W2", "b1", "b2"))
    Z = X @ W1
    Z = Z if b1 is None else Z + b1
    A, slope = _act_and_slope(Z, act)
    U = None if W1u is None else X @ W1u
    H = A if U is None else A * U
    Y = H @ W2
    out = {"Y": Y if b2 is None else Y + b2}
    if train:
        dY = f(s["dY"])
        dH = dY @ W2.t()
        dZ = dH * slope if U is None else dH * U * slope
        out["dX"] = dZ @ W1.t()
        out["dW1"] = X.t() @ dZ
        if U is not None:
            dU = dH * A
            out["dX"] = out["dX"] + dU @ W1u.t()
            out["dW1u"] = X.t() @ dU
        if b1 is not None:
            out["db1"] = dZ.sum(0)
        out["dW2"] = H.t() @ dY
        if b2 is not None:
            out["db2"] = dY.sum(0)
    return {k: v.to(dt) for k, v in out.items()}


# ---------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    if case["kind"] == "clip":
        wide = [x.double() for x in _draw_grads(case, seed)[0].values()]
        norm = math.sqrt(math.fsum(float(torch.dot(x, x)) for x in wide))
        factor = min(1.0, 1.0 / (norm + 1e-6))
        names = [k for k, t in DTYPES.items() if any(t is v for v in _kinds(case, len(_sizes(case))))]
        return {"norm": torch.tensor([norm], dtype=torch.float64), **{k: x.mul_(factor) for k, x in zip(names, wide)}}
    s = {k: None if v is None else v.double() for k, v in _draw_ffn(case, seed).items()}
    act, zero = case["act"], torch.zeros((), dtype=torch.float64, device="cuda")
    pre = torch.matmul(s["X"], s["W1"]).add_(zero if s["b1"] is None else s["b1"])
    if act == "swiglu":
        e = torch.exp(-pre)
        value, slope = pre / (1 + e), (1 + e + pre * e) / (1 + e) ** 2
    elif act == "gelu_erf":
        below = torch.erfc(-pre / math.sqrt(2)) / 2        # the normal distribution's share below z
        value, slope = pre * below, below + pre * torch.exp(-pre ** 2 / 2) / math.sqrt(2 * math.pi)
    else:
        k = math.sqrt(8 / math.pi)                          # (1 + tanh v) / 2 = 1 / (1 + exp(-2 v))
        below = 1 / (1 + torch.exp(-k * (pre + 0.044715 * pre ** 3)))
        value, slope = pre * below, below + pre * below * (1 - below) * k * (1 + 0.134145 * pre ** 2)
    up = None if s["W1u"] is None else torch.matmul(s["X"], s["W1u"])
    hidden = value if up is None else value * up
    out = {"Y": torch.matmul(hidden, s["W2"]).add_(zero if s["b2"] is None else s["b2"])}
    if case["kind"] == "train":
        back = torch.einsum("td,md->tm", s["dY"], s["W2"])
        through = back * slope * (1 if up is None else up)
        out["dX"] = torch.einsum("tm,dm->td", through, s["W1"])
        out["dW1"] = torch.einsum("td,tm->dm", s["X"], through)
        if up is not None:
            out["dX"] += torch.einsum("tm,dm->td", back * value, s["W1u"])
            out["dW1u"] = torch.einsum("td,tm->dm", s["X"], back * value)
        out["dW2"] = torch.einsum("tm,td->md", hidden, s["dY"])
        if s["b1"] is not None:
            out["db1"], out["db2"] = torch.einsum("tm->m", through), torch.einsum("td->d", s["dY"])
    return out
