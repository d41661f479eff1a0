"""More of the library's operators, as they are measured: the update of a list of matrices by orthogonalised momentum,
the orthogonalisation alone, low-rank adapters of many requests beside a shared projection, and their gradients.

`run` computes a case in its plain form (elementary torch operations in 32 bits, rounded once at the end), or with
`own` through the library's entry points; `exact` is the same result from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
ITERATIONS = 5
BETA = 0.95


# ---------------------------------------------------------------------------------------------------- the cases
def _matrices(name, kind, shapes, dtype):
    """kind: "muon" (the whole update) or "orthogonalize"; shapes: "<rows>x<cols>x<count>", joined by "+"."""
    return {"name": name, "kind": kind, "shapes": shapes, "dtype": dtype}


def _adapters(name, kind, inner, outer, T, n, r, dtype, order, shared, seed_index=1):
    """kind: "forward" or "backward"; order: how the tokens' adapters lie in the batch ("segments": request after request;
    "single": a token each; "mixed": segments, then single tokens); shared: what the adapters are beside ("weight": the
    projection's product is part of the call; "base": its result is given)."""
    return {"name": name, "kind": kind, "in": inner, "out": outer, "T": T, "n": n, "r": r, "dtype": dtype, "order": order,
            "shared": shared, "seed_index": seed_index}


def listed():
    return [
        # the three matrices of a 4096 x 11008 gated layer
        _matrices("muon gated layer", "muon", "4096x11008x2+11008x4096x1", "bf16"),
        # all matrices of a 24-layer stack of 1024 x 4096 layers
        _matrices("muon 24 layers", "muon", "1024x4096x24+4096x1024x24", "bf16"),
        # the factors of sixteen adapters of rank 16
        _matrices("muon adapter factors", "muon", "4096x16x16+16x11008x16", "bf16"),
        # a 32-bit gated layer
        _matrices("muon f32 layer", "muon", "1024x2752x2+2752x1024x1", "f32"),
        # one small matrix: the latency of the launches
        _matrices("orthogonalize 256x1024", "orthogonalize", "256x1024x1", "bf16"),
        # widths that fill no tile: neurons left over after others were removed
        _matrices("orthogonalize ragged", "orthogonalize", "1000x2731x2+2731x1000x1", "bf16"),
        # a generation step of 32 requests, each with its own adapter
        _adapters("adapters 32 requests", "forward", 4096, 11008, 32, 48, 16, "bf16", "single", "weight"),
        # prompts of many requests and the next tokens of others in one batch
        _adapters("adapters prompts", "forward", 4096, 11008, 4096, 24, 32, "bf16", "mixed", "weight"),
        # beside a layer whose output is already there, a ragged batch
        _adapters("adapters beside a layer", "forward", 1000, 1000, 777, 6, 8, "bf16", "segments", "base"),
        # 32-bit layers
        _adapters("adapters f32", "forward", 1024, 2752, 300, 5, 12, "f32", "mixed", "weight"),
        # fine-tuning one adapter of rank 64 on a 2048-token sequence
        _adapters("adapter training", "backward", 4096, 11008, 2048, 1, 64, "bf16", "segments", "weight"),
        # several fine-tunes in one batch
        _adapters("adapters training ragged", "backward", 1024, 4096, 1000, 7, 24, "bf16", "segments", "weight"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["muon", "orthogonalize", "forward", "forward", "backward"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("muon", "orthogonalize"):
        limit = 0.7 * max(_flops(c) for c in listed()) * (1.0 if dtype == "bf16" else 0.1)
        while True:
            parts = []
            for _ in range(rng.choice([1, 1, 2, 3])):
                rows, cols = _log_int(rng, 8, 8192), _log_int(rng, 8, 11008)
                parts.append("%dx%dx%d" % (rows, cols, _log_int(rng, 1, 32)))
            case = {"kind": kind, "shapes": "+".join(parts), "dtype": dtype}
            if _flops(case) <= limit and sum(r * c for r, c in _shapes(case)) <= 2e8:
                return case
    big = 1.0 if dtype == "bf16" else 0.4     # 32-bit layers stay smaller
    order = rng.choice(["segments", "single", "mixed"])
    case = {"kind": kind, "in": _log_int(rng, 64, int(8192 * big)), "out": _log_int(rng, 64, int(11008 * big)),
            "T": _log_int(rng, 1, 64 if order == "single" else int(8192 * big)), "n": _log_int(rng, 1, 64), "r": _log_int(rng, 4, 128),
            "dtype": dtype, "order": order, "shared": rng.choice(["weight", "weight", "base"]), "seed_index": rng.randrange(1, 1 << 30)}
    if dtype == "bf16" and rng.random() < 0.75:     # most widths and ranks are whole vectors of 16 bytes
        for k in ("in", "out", "r"):
            case[k] = (case[k] + 7) // 8 * 8
    return case


def _shapes(case):
    """(rows, cols) of every matrix of a case, from its text."""
    out = []
    for part in case["shapes"].split("+"):
        rows, cols, count = (int(v) for v in part.split("x"))
        out += [(rows, cols)] * count
    return out


def _index(case):
    """The adapter of every token (-1: the request has none)."""
    r, T, n = random.Random(case["seed_index"]), case["T"], case["n"]
    pick = lambda: -1 if n > 2 and r.random() < 0.1 else r.randrange(n)  # noqa: E731
    single = T if case["order"] == "single" else T // 16 if case["order"] == "mixed" else 0
    out = []
    while len(out) < T - single:
        out += [pick()] * max(1, int((T - single) / max(1, n) * math.exp(r.gauss(0.0, 0.7))))
    return out[:T - single] + [pick() for _ in range(single)]


def _flops(case):
    if "shapes" in case:
        total = 0.0
        for rows, cols in _shapes(case):
            p, q = min(rows, cols), max(rows, cols)
            total += ITERATIONS * (3.0 * p * p * q + 1.0 * p * p * p)      # two of the three products are symmetric
        return total
    T, k, m, r = case["T"], case["in"], case["out"], case["r"]
    active = sum(1 for i in _index(case) if i >= 0)
    shared = 2.0 * T * k * m if case["shared"] == "weight" else 0.0
    return shared + 2.0 * active * r * (k + m) * (1 if case["kind"] == "forward" else 3)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if "shapes" in case:
        elements = sum(rows * cols for rows, cols in _shapes(case))
        # weights, gradients and momentum are read, weights and momentum written; or one matrix to another
        return {"bytes": float(elements * (3 * e + 8 if case["kind"] == "muon" else 2 * e)), "flops": _flops(case)}
    T, k, m, r = case["T"], case["in"], case["out"], case["r"]
    used = len(set(i for i in _index(case) if i >= 0))
    factors = used * r * (k + m) * e
    weight = k * m * e if case["shared"] == "weight" else (m if case["kind"] == "forward" else k) * T * e
    if case["kind"] == "forward":
        return {"bytes": float(e * T * (k + m) + weight + factors + 4 * T), "flops": _flops(case)}
    gradients = case["n"] * r * (k + m) * e
    return {"bytes": float(e * T * (2 * k + m) + weight + factors + gradients + 4 * T), "flops": _flops(case)}


# ---------------------------------------------------------------------------------------------------- inputs
def _draw_matrices(case, seed):
    """Gradients as a batch leaves them: a few strong directions and noise; momentum of the steps before it with some of
    the same directions."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 11)
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    dt, muon = DTYPES[case["dtype"]], case["kind"] == "muon"
    out = {"G": [], "M": [], "W": []}
    for rows, cols in _shapes(case):
        rank = max(1, min(rows, cols) // 16)
        strength = torch.exp(-3.0 * torch.arange(rank, device="cuda") / rank)
        left, right = randn(rows, rank) * strength, randn(rank, cols)
        out["G"].append((1e-3 * (left @ right + 0.5 * randn(rows, cols))).to(dt))
        if muon:
            out["M"].append(4e-3 * (left @ (0.7 * right + 0.7 * randn(rank, cols)) + 0.3 * randn(rows, cols)))
            out["W"].append((0.02 * randn(rows, cols)).to(dt))
    return out


def _views(case, flat):
    shapes = _shapes(case)
    return [v.view(s) for v, s in zip(torch.split(flat, [r * c for r, c in shapes]), shapes)]


def _joined(matrices):
    return torch.cat([v.reshape(-1) for v in matrices])


def _rates(rows, cols):
    """step and decay of one matrix: the learning rate times what makes the update's elements as large as 0.2, and times the decay."""
    return 0.01 * 0.2 * math.sqrt(max(rows, cols)), 0.01 * 0.1


def _draw_adapters(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + case["in"] * 31 + case["out"] * 17 + case["T"])
    dt, T, k, m, n, r = DTYPES[case["dtype"]], case["T"], case["in"], case["out"], case["n"], case["r"]
    new = lambda scale, *shape: (torch.randn(*shape, generator=g, device="cuda") * scale).to(dt)  # noqa: E731
    forward, weight = case["kind"] == "forward", case["shared"] == "weight"
    return {
        "X": new(1.0, T, k),
        "W": new(k ** -0.5, k, m) if weight else None,
        "b": new(0.1, m) if weight and forward else None,
        "base": None if weight else new(1.0, T, m) if forward else new(1e-3, T, k),
        "A": new(k ** -0.5, n, k, r),
        "B": new(0.5 * r ** -0.5, n, r, m),
        "scale": torch.rand(n, generator=g, device="cuda") + 0.5,
        "index": torch.tensor(_index(case), dtype=torch.int32, device="cuda"),
        "dY": None if forward else new(1e-3, T, m),
    }


_library = {}


def _context():
    """The library's context, one to a process."""
    if "ctx" not in _library:
        from paper_2401_04044_b200 import Context
        _library["ctx"] = Context(0)
    return _library["ctx"]


def prepare(case, seed):
    """The inputs; with `own` also what a program that uses the library keeps between calls: the context with its
    workspace, the buffers for results, and the list that names the matrices.  Nothing is computed from the inputs."""
    if "shapes" in case:
        state = {"case": case, **_draw_matrices(case, seed)}
        if own:
            ctx, muon = _context(), case["kind"] == "muon"
            # results lie in one buffer, matrix after matrix without gaps (so that some start off a 16-byte boundary)
            whole = sum(r * c for r, c in _shapes(case))
            state["out"] = torch.empty(whole, dtype=DTYPES[case["dtype"]], device="cuda")
            if muon:
                state["out_M"] = torch.empty(whole, dtype=torch.float32, device="cuda")
                rates = [_rates(*s) for s in _shapes(case)]
                state["list"] = ctx.muon_list(state["W"], state["G"], state["M"], [s for s, _ in rates], [d for _, d in rates],
                                              out_weights=_views(case, state["out"]), out_momenta=_views(case, state["out_M"]))
            else:
                state["list"] = ctx.orthogonal_list(state["G"], _views(case, state["out"]))
            ctx.ensure_workspace(ctx.muon_workspace_size(state["list"]))
        return state
    state = {"case": case, **_draw_adapters(case, seed)}
    if own:
        from paper_2401_04044_b200 import Projection
        ctx = _context()
        state["projection"] = Projection(case["in"], case["out"], DTYPES[case["dtype"]])
        ctx.ensure_workspace(ctx.adapter_workspace_size(state["projection"], case["n"], case["r"], case["T"]))
        if case["kind"] == "forward":
            state["Y"] = torch.empty(case["T"], case["out"], dtype=DTYPES[case["dtype"]], device="cuda")
        else:
            state["grads"] = {"d" + k: torch.empty_like(state[k]) for k in ("X", "A", "B")}
    else:      # adapter by adapter the rows of the batch that use it
        index = _index(case)
        state["rows"] = [(i, torch.tensor([t for t, j in enumerate(index) if j == i], device="cuda")) for i in sorted(set(index) - {-1})]
    return state


# ---------------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "muon":
        return _plain_muon(state)
    if kind == "orthogonalize":
        return {"O": _joined([_plain_orthogonal(g.float()).to(g.dtype) for g in state["G"]])}
    return _plain_forward(state) if kind == "forward" else _plain_backward(state)


def _run_own(s):
    ctx, kind = _context(), s["case"]["kind"]
    if kind == "muon":
        ctx.muon_step(s["list"], BETA)
        return {"W": s["out"], "M": s["out_M"]}
    if kind == "orthogonalize":
        ctx.orthogonalize(s["list"])
        return {"O": s["out"]}
    if kind == "forward":
        ctx.adapter_forward(s["projection"], s["X"], s["A"], s["B"], s["index"], s["Y"], W=s["W"], b=s["b"], base=s["base"], scale=s["scale"])
        return {"Y": s["Y"]}
    ctx.adapter_backward(s["projection"], s["X"], s["A"], s["B"], s["index"], s["dY"], W=s["W"], base=s["base"], scale=s["scale"], **s["grads"])
    return dict(s["grads"])


def _plain_orthogonal(u):
    a, b, c = COEFFICIENTS
    tall = u.shape[0] > u.shape[1]
    x = u.t() if tall else u
    x = x / (torch.sqrt((x * x).sum()) + 1e-7)
    for _ in range(ITERATIONS):
        s = x @ x.t()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if tall else x


def _plain_muon(s):
    weights, momenta = [], []
    for w, g, m in zip(s["W"], s["G"], s["M"]):
        step, decay = _rates(*w.shape)
        momentum = BETA * m + g.float()
        o = _plain_orthogonal(g.float() + BETA * momentum)
        weights.append(((1.0 - decay) * w.float() - step * o).to(w.dtype))
        momenta.append(momentum)
    return {"W": _joined(weights), "M": _joined(momenta)}


def _plain_forward(s):
    f = lambda t: None if t is None else t.float()  # noqa: E731
    X, A, B = f(s["X"]), f(s["A"]), f(s["B"])
    Y = f(s["base"]).clone() if s["W"] is None else X @ f(s["W"])
    if s["b"] is not None:
        Y = Y + f(s["b"])
    for i, rows in s["rows"]:
        Y[rows] += s["scale"][i] * ((X[rows] @ A[i]) @ B[i])
    return {"Y": Y.to(s["X"].dtype)}


def _plain_backward(s):
    f = lambda t: None if t is None else t.float()  # noqa: E731
    X, A, B, dY, dt = f(s["X"]), f(s["A"]), f(s["B"]), f(s["dY"]), s["X"].dtype
    dX = f(s["base"]).clone() if s["W"] is None else dY @ f(s["W"]).t()
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    for i, rows in s["rows"]:
        x, d = X[rows], s["scale"][i] * dY[rows]
        inner = d @ B[i].t()
        dX[rows] += inner @ A[i].t()
        dA[i] = x.t() @ inner
        dB[i] = (x @ A[i]).t() @ d
    return {"dX": dX.to(dt), "dA": dA.to(dt), "dB": dB.to(dt)}


# ---------------------------------------------------------------------------------------------------- 64 bits
def _exact_orthogonal(u):
    """On the matrix as it lies: p(X X^T) X = X p(X^T X), whichever square is smaller."""
    x = u.div(torch.linalg.vector_norm(u) + 1e-7)
    a, b, c = COEFFICIENTS
    for _ in range(ITERATIONS):
        if x.shape[0] <= x.shape[1]:
            gram = torch.einsum("ik,jk->ij", x, x)
            x = torch.addmm(x, torch.addmm(gram, gram, gram, beta=b, alpha=c), x, beta=a)
        else:
            gram = torch.einsum("ki,kj->ij", x, x)
            x = torch.addmm(x, x, torch.addmm(gram, gram, gram, beta=b, alpha=c), beta=a)
    return x


def exact(case, seed):
    if "shapes" in case:
        s = _draw_matrices(case, seed)
        if case["kind"] == "orthogonalize":
            return {"O": _joined([_exact_orthogonal(g.double()) for g in s["G"]])}
        weights, momenta = [], []
        for w, g, m in zip(s["W"], s["G"], s["M"]):
            step, decay = _rates(*w.shape)
            new = m.double().mul_(BETA).add_(g.double())
            weights.append(w.double().mul_(1.0 - decay).sub_(_exact_orthogonal(new.mul(BETA).add_(g.double())), alpha=step))
            momenta.append(new)
        return {"W": _joined(weights), "M": _joined(momenta)}
    s = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in _draw_adapters(case, seed).items()}
    X, A, B, index = s["X"], s["A"], s["B"], s["index"].long()
    if case["kind"] == "forward":
        Y = s["base"].clone() if s["W"] is None else torch.einsum("tk,km->tm", X, s["W"]).add_(s["b"])
        for i in range(case["n"]):
            mine = index.eq(i)
            Y[mine] += torch.linalg.multi_dot([X[mine], A[i], B[i]]).mul_(s["scale"][i]) if bool(mine.any()) else 0.0
        return {"Y": Y}
    dY = s["dY"]
    dX = s["base"].clone() if s["W"] is None else torch.einsum("tm,km->tk", dY, s["W"])
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    for i in range(case["n"]):
        mine = index.eq(i)
        if bool(mine.any()):
            # the gradient of the factors' product, taken apart
            outer = torch.einsum("tk,tm->km", X[mine], dY[mine]).mul_(s["scale"][i])
            dA[i], dB[i] = torch.einsum("km,rm->kr", outer, B[i]), torch.einsum("kr,km->rm", A[i], outer)
            dX[mine] += torch.einsum("tm,km->tk", dY[mine], torch.matmul(A[i], B[i])).mul_(s["scale"][i])
    return {"dX": dX, "dA": dA, "dB": dB}
