"""Low-rank adapters beside a shared projection, and their gradients, against plain implementations in 64 bits on the same
stored inputs.

Tolerances.  bf16: X A_i (dY B_i^T) is rounded to bf16 before the second product, the shared product may be rounded before
the adapters' part is added, and the result is rounded: three independent roundings of an rms of 0.43 2^-8 at most, 2.9e-3 of
the norm; 4e-3 is asked for.  fp32: 1e-5, as everywhere in the library.  Single elements: 8 times that of the largest."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TOL = {"bf16": 4e-3, "f32": 1e-5}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ctx():
    from paper_2401_04044_b200 import Context, build
    build.build()
    c = Context(0)
    c.ensure_workspace(1 << 20)
    yield c
    c.close()


def index_of(order, T, n, seed):
    r = np.random.default_rng(seed)
    if order == "none":
        return np.full(T, -1, np.int32)
    if order == "one":
        return np.full(T, n - 1, np.int32)
    if order == "segments":
        out = np.sort(r.integers(-1, n, T))
        return out.astype(np.int32)
    return r.integers(-1, n, T).astype(np.int32)


def draw(dtype, k, m, T, n, r, order="mixed", shared="weight", seed=0, bias=True, scaled=True):
    g = torch.Generator().manual_seed(seed * 977 + k + 3 * m + 7 * T + n)
    new = lambda s, *shape: (torch.randn(*shape, generator=g) * s).to(DT[dtype])  # noqa: E731
    return {"X": new(1.0, T, k), "W": new(k ** -0.5, k, m) if shared == "weight" else None,
            "b": new(0.2, m) if shared == "weight" and bias else None, "base": new(1.0, T, m) if shared == "base" else None,
            "base_dX": new(0.01, T, k) if shared == "base" else None,
            "A": new(k ** -0.5, n, k, r), "B": new(r ** -0.5, n, r, m), "dY": new(0.01, T, m),
            "scale": torch.rand(n, generator=g) * 2 - 0.5 if scaled else None, "index": torch.from_numpy(index_of(order, T, n, seed + T))}


def reference(L):
    f = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    X, W, A, B, dY, index = f(L["X"]), f(L["W"]), f(L["A"]), f(L["B"]), f(L["dY"]), L["index"].numpy()
    Y = X @ W if W is not None else f(L["base"]).copy() if L["base"] is not None else np.zeros_like(dY)
    if L["b"] is not None:
        Y = Y + f(L["b"])
    dX = dY @ W.T if W is not None else f(L["base_dX"]).copy() if L["base_dX"] is not None else np.zeros_like(X)
    dA, dB = np.zeros_like(A), np.zeros_like(B)
    for i in range(A.shape[0]):
        t = np.nonzero(index == i)[0]
        s = 1.0 if L["scale"] is None else float(L["scale"][i])
        Y[t] += s * X[t] @ A[i] @ B[i]
        d = s * dY[t] @ B[i].T
        dX[t] += d @ A[i].T
        dA[i] = X[t].T @ d
        dB[i] = s * (X[t] @ A[i]).T @ dY[t]
    return {"Y": Y, "dX": dX, "dA": dA, "dB": dB}


def guarded(shape, dt):
    n = int(np.prod(shape))
    flat = torch.full(((n + 63) // 32 * 32 + 64,), -7.0, dtype=dt, device="cuda")
    return flat, flat[32:32 + n].view(*shape)


def run(ctx, L, dtype, want=("Y", "dX", "dA", "dB"), stream=None, in_place=False):
    from paper_2401_04044_b200 import Projection
    D = {k: None if v is None else v.cuda() for k, v in L.items()}
    (T, k), (n, _, r), m = L["X"].shape, L["A"].shape, L["B"].shape[2]
    p = Projection(k, m, DT[dtype])
    ctx.ensure_workspace(ctx.adapter_workspace_size(p, n, r, T))
    shapes = {"Y": (T, m), "dX": (T, k), "dA": (n, k, r), "dB": (n, r, m)}
    bufs = {o: guarded(shapes[o], DT[dtype]) for o in want}
    if in_place:
        for o, base in (("Y", "base"), ("dX", "base_dX")):
            if o in bufs:
                bufs[o][1].copy_(D[base])
                D[base] = bufs[o][1]
    torch.cuda.synchronize()
    if "Y" in want:
        ctx.adapter_forward(p, D["X"], D["A"], D["B"], D["index"], bufs["Y"][1], W=D["W"], b=D["b"], base=D["base"], scale=D["scale"], stream=stream)
    grads = {o: b[1] for o, b in bufs.items() if o != "Y"}
    if grads:
        ctx.adapter_backward(p, D["X"], D["A"], D["B"], D["index"], D["dY"], W=D["W"], base=D["base_dX"], scale=D["scale"], stream=stream, **grads)
    ctx.poll(stream)
    torch.cuda.synchronize()
    for o, (flat, t) in bufs.items():
        assert (flat[:32] == -7).all() and (flat[32 + t.numel():] == -7).all(), f"{o}: written outside the tensor"
    return {o: b[1].cpu() for o, b in bufs.items()}


def check(got, L, dtype):
    ref = reference(L)
    for o, v in got.items():
        x, r = v.double().numpy(), ref[o]
        norm, top = np.linalg.norm(r), np.abs(r).max()
        if norm == 0:
            assert (x == 0).all(), o
            continue
        err, big = np.linalg.norm(x - r) / norm, np.abs(x - r).max() / top
        assert err <= TOL[dtype] and big <= 8 * TOL[dtype], f"{o}: {err:.2e} of the norm (<= {TOL[dtype]}), {big:.2e} of the largest element"


SIZES = [  # k, m, T, n, r
    (8, 8, 1, 1, 1), (64, 64, 1, 1, 8), (64, 128, 2, 5, 16), (200, 72, 7, 3, 8), (256, 1024, 33, 40, 16), (520, 264, 130, 9, 24),
    (136, 520, 257, 4, 64), (1000, 1000, 300, 6, 8), (328, 96, 515, 2, 128), (264, 392, 700, 70, 40), (1024, 512, 64, 64, 32),
    (2048, 136, 5, 2, 96), (77, 131, 50, 3, 5), (131, 77, 200, 4, 70), (33, 1, 9, 2, 3), (1, 40, 20, 3, 127)]


@pytest.mark.parametrize("shared", ["weight", "base", "alone"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k,m,T,n,r", SIZES)
def test_forward_and_gradients(ctx, dtype, k, m, T, n, r, shared):
    L = draw(dtype, k, m, T, n, r, shared=shared, order="segments" if T % 2 else "mixed")
    check(run(ctx, L, dtype), L, dtype)


@pytest.mark.parametrize("order", ["none", "one", "segments", "mixed"])
@pytest.mark.parametrize("dtype,k,m,T,n,r", [("bf16", 264, 520, 300, 7, 16), ("bf16", 512, 256, 1, 3, 8), ("f32", 100, 60, 70, 5, 12)])
def test_orders(ctx, dtype, k, m, T, n, r, order):
    L = draw(dtype, k, m, T, n, r, order=order, seed=4, bias=False, scaled=order != "one")
    check(run(ctx, L, dtype), L, dtype)


@pytest.mark.parametrize("dtype,k,m,T,n,r,order", [("bf16", 1024, 2816, 3000, 11, 32, "segments"), ("bf16", 2048, 1000, 1500, 1, 64, "one"),
                                                   ("bf16", 640, 2000, 1100, 300, 16, "mixed"), ("f32", 640, 1111, 1000, 5, 20, "segments")])
def test_many_tiles(ctx, dtype, k, m, T, n, r, order):
    L = draw(dtype, k, m, T, n, r, order=order, seed=3)
    check(run(ctx, L, dtype), L, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_alone_and_together_have_the_same_bits(ctx, dtype):
    L = draw(dtype, 200, 328, 400, 5, 24, order="segments", seed=6)
    whole = run(ctx, L, dtype)
    for want in (("dX",), ("dA",), ("dB",), ("dA", "dB"), ("dX", "dB")):
        for o, v in run(ctx, L, dtype, want=want).items():
            assert torch.equal(v, whole[o]), o


@pytest.mark.parametrize("dtype,k,m,T,n,r", [("bf16", 264, 520, 300, 7, 16), ("bf16", 77, 91, 40, 7, 9), ("f32", 60, 100, 20, 3, 8)])
def test_added_in_place(ctx, dtype, k, m, T, n, r):
    L = draw(dtype, k, m, T, n, r, shared="base", order="segments", seed=8)
    a, b = run(ctx, L, dtype), run(ctx, L, dtype, in_place=True)
    assert all(torch.equal(a[o], b[o]) for o in a)
    check(b, L, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_adapter_behind_the_last_counts_as_none_and_is_reported(ctx, dtype):
    from paper_2401_04044_b200 import FFSplitError
    L = draw(dtype, 64, 96, 40, 3, 8, seed=9)
    L["index"][17] = 3
    L["index"][20] = 2 ** 31 - 1
    L["index"][21] = -2 ** 31
    with pytest.raises(FFSplitError) as e:
        run(ctx, L, dtype)
    assert e.value.code == 11
    fixed = {**L, "index": torch.where((L["index"] >= 3) | (L["index"] < 0), torch.full_like(L["index"], -1), L["index"])}
    from paper_2401_04044_b200 import Projection
    p, D = Projection(64, 96, DT[dtype]), {k: None if v is None else v.cuda() for k, v in L.items()}
    Y = torch.empty(40, 96, dtype=DT[dtype], device="cuda")
    dA = torch.empty_like(D["A"])
    ctx.adapter_forward(p, D["X"], D["A"], D["B"], D["index"], Y, W=D["W"], b=D["b"], scale=D["scale"])
    ctx.adapter_backward(p, D["X"], D["A"], D["B"], D["index"], D["dY"], W=D["W"], scale=D["scale"], dA=dA)
    with pytest.raises(FFSplitError):
        ctx.poll()
    ctx.poll()
    check({"Y": Y.cpu(), "dA": dA.cpu()}, fixed, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_token_that_is_not_finite_reaches_its_own_row_and_adapter_only(ctx, dtype):
    L = draw(dtype, 72, 136, 90, 4, 16, order="mixed", seed=11)
    t = int(np.nonzero(L["index"].numpy() == 2)[0][0])
    clean = run(ctx, L, dtype)
    L["X"][t, 5] = float("nan")
    got = run(ctx, L, dtype, want=("Y", "dA", "dB"))
    rows = [i for i in range(90) if i != t]
    assert torch.equal(got["Y"][rows], clean["Y"][rows]) and torch.isnan(got["Y"][t]).all()
    for o in ("dA", "dB"):
        assert torch.equal(got[o][[0, 1, 3]], clean[o][[0, 1, 3]]), o
    assert torch.isnan(got["dB"][2]).all() and torch.isnan(got["dA"][2][5]).all()


def test_an_adapter_nobody_uses_may_hold_anything(ctx):
    L = draw("bf16", 72, 136, 90, 4, 16, order="mixed", seed=12)
    L["index"][L["index"] == 1] = 0
    clean = run(ctx, L, "bf16")
    L["A"][1], L["B"][1] = float("nan"), float("inf")
    got = run(ctx, L, "bf16")
    assert all(torch.equal(got[o], clean[o]) for o in got)


def test_refusals(ctx):
    from paper_2401_04044_b200 import FFSplitError, Projection
    L = {k: None if v is None else v.cuda() for k, v in draw("bf16", 64, 96, 10, 3, 8).items()}
    p = Projection(64, 96, torch.bfloat16)
    ctx.ensure_workspace(ctx.adapter_workspace_size(p, 3, 8, 10))
    Y = torch.empty(10, 96, dtype=torch.bfloat16, device="cuda")

    def forward(code, **kw):
        a = {"X": L["X"], "A": L["A"], "B": L["B"], "index": L["index"], "Y": Y, "W": L["W"], **kw}
        with pytest.raises(FFSplitError) as e:
            ctx.adapter_forward(p, a.pop("X"), a.pop("A"), a.pop("B"), a.pop("index"), a.pop("Y"), **a)
        assert e.value.code == code

    forward(4, X=L["X"].float())
    forward(2, X=L["X"][:, :32])
    forward(2, A=L["A"][0])
    forward(2, B=L["B"][:2])
    forward(4, index=L["index"].long())
    forward(2, index=L["index"][:5])
    forward(1, index=L["index"].cpu())
    forward(1, base=Y.clone())
    forward(1, W=None, b=L["b"])
    forward(4, scale=L["scale"].bfloat16())
    forward(3, X=torch.empty(641, dtype=torch.bfloat16, device="cuda")[1:].view(10, 64))
    forward(2, A=torch.zeros(3, 64, 136, dtype=torch.bfloat16, device="cuda"), B=torch.zeros(3, 136, 96, dtype=torch.bfloat16, device="cuda"))
    forward(2, A=torch.zeros(3, 64, 0, dtype=torch.bfloat16, device="cuda"), B=torch.zeros(3, 0, 96, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(FFSplitError) as e:
        ctx.adapter_backward(p, L["X"], L["A"], L["B"], L["index"], L["dY"], W=L["W"])
    assert e.value.code == 1
    kept = ctx._ws
    ctx.set_workspace(torch.empty(65536, dtype=torch.uint8, device="cuda"))
    forward(5)
    ctx.set_workspace(kept)


def test_other_stream_and_captured_replay(ctx):
    """A captured call that is replayed takes the tokens and the adapters of each replay."""
    from paper_2401_04044_b200 import Projection
    Ls = [draw("bf16", 128, 264, 48, 6, 16, seed=s) for s in (20, 21, 22)]
    p = Projection(128, 264, torch.bfloat16)
    D = {k: None if v is None else v.cuda() for k, v in Ls[0].items()}
    ctx.ensure_workspace(ctx.adapter_workspace_size(p, 6, 16, 48))
    Y = torch.empty(48, 264, dtype=torch.bfloat16, device="cuda")
    dA, dB, dX = torch.empty_like(D["A"]), torch.empty_like(D["B"]), torch.empty_like(D["X"])

    def call():
        ctx.adapter_forward(p, D["X"], D["A"], D["B"], D["index"], Y, W=D["W"], b=D["b"], scale=D["scale"])
        ctx.adapter_backward(p, D["X"], D["A"], D["B"], D["index"], D["dY"], W=D["W"], scale=D["scale"], dX=dX, dA=dA, dB=dB)

    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    check({"Y": Y.cpu(), "dX": dX.cpu(), "dA": dA.cpu(), "dB": dB.cpu()}, Ls[0], "bf16")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for L in Ls[1:]:
        for k, v in L.items():
            if v is not None:
                D[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        check({"Y": Y.cpu(), "dX": dX.cpu(), "dA": dA.cpu(), "dB": dB.cpu()}, L, "bf16")
    ctx.poll()


# (the last two: outputs of more than 2^25 elements, whose adapters are taken along in the shared product)
@pytest.mark.parametrize("dtype,T,n,k,m", [("bf16", 40, 4, 264, 520), ("bf16", 300, 4, 264, 520), ("bf16", 700, 20, 264, 520), ("f32", 40, 4, 60, 100),
                                           ("f32", 300, 4, 60, 100), ("bf16", 4200, 4, 264, 8200), ("bf16", 4201, 3, 8200, 264)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_broken_adapter_reaches_its_own_tokens_only(ctx, dtype, T, n, k, m, value):
    """Zero times an infinity is NaN: the rows of other requests in the same tile must not meet a factor that holds one."""
    L = draw(dtype, k, m, T, n, 16, order="mixed", seed=13)
    clean = run(ctx, L, dtype)
    bad = L["index"] == 2
    L["A"][2, 5, 3], L["B"][2, 1, 7] = value, value
    got = run(ctx, L, dtype)
    for o in ("Y", "dX"):
        assert torch.equal(got[o][~bad], clean[o][~bad]), o
    assert not torch.isfinite(got["Y"][bad][:, 7]).any() and not torch.isfinite(got["dX"][bad][:, 5]).any()
    others = [i for i in range(n) if i != 2]
    assert torch.equal(got["dA"][others], clean["dA"][others]) and torch.equal(got["dB"][others], clean["dB"][others])
    # columns that the broken element does not reach
    L["A"][2, 5, 3] = 0.0
    once = run(ctx, L, dtype, want=("Y",))["Y"]
    keep = [c for c in range(m) if c != 7]
    L["B"][2, 1, 7] = 0.0
    ref = reference(L)["Y"][:, keep]
    x = once[:, keep].double().numpy()
    assert np.linalg.norm(x - ref) <= TOL[dtype] * np.linalg.norm(ref)


@pytest.mark.parametrize("shared", ["weight", "base"])
@pytest.mark.parametrize("T,n,r,k,m", [(1024, 40, 16, 640, 776), (777, 40, 72, 640, 776), (513, 12, 128, 640, 776), (4300, 40, 16, 648, 8008), (4201, 12, 72, 8200, 456),
                                       (4111, 12, 128, 712, 8200), (6500, 1, 24, 5201, 257)])
def test_tiles_with_few_and_with_many_adapters_in_one_batch(ctx, T, n, r, k, m, shared):
    """Of the first rows all of one adapter, of the middle some without any, of the rest each another one."""
    L = draw("bf16", k, m, T, n, r, order="mixed", shared=shared, seed=14)
    L["index"][:250] = n - 1
    L["index"][250:500] = -1
    L["index"][300:310] = 0
    check(run(ctx, L, "bf16"), L, "bf16")


def test_more_adapters_than_the_tensor_cores_tiles_allow(ctx):
    """65535 adapters and 70000 tokens: the batch stays on the CUDA cores."""
    L = draw("bf16", 8, 16, 70000, 65535, 1, order="mixed", seed=15)
    D = {k: None if v is None else v.double() for k, v in L.items() if k not in ("index", "scale", "base", "base_dX")}
    got = run(ctx, L, "bf16")
    i = L["index"].long()
    used, at = (i >= 0).double().unsqueeze(1), i.clamp_min(0)
    s = L["scale"].double()[at].unsqueeze(1) * used
    A, B = D["A"][at, :, 0], D["B"][at, 0, :]
    P, G = s * (D["X"] * A).sum(1, keepdim=True), s * (D["dY"] * B).sum(1, keepdim=True)
    ref = {"Y": D["X"] @ D["W"] + D["b"] + P * B, "dX": D["dY"] @ D["W"].t() + G * A,
           "dA": torch.zeros_like(D["A"][:, :, 0]).index_add_(0, at, G * D["X"]).unsqueeze(2),
           "dB": torch.zeros_like(D["B"][:, 0, :]).index_add_(0, at, P * D["dY"]).unsqueeze(1)}
    for o, v in got.items():
        assert float((v.double() - ref[o]).norm() / ref[o].norm()) <= TOL["bf16"], o


@pytest.mark.parametrize("dtype,T", [("f32", 3), ("bf16", 3), ("bf16", 70)])
@pytest.mark.parametrize("k,m", [(5, (1 << 21) + 35), ((1 << 21) + 35, 5)])
def test_more_columns_than_a_grid_has_rows_of_blocks(ctx, dtype, T, k, m):
    L = draw(dtype, k, m, T, 2, 3, shared="base")
    check(run(ctx, L, dtype, in_place=True), L, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shared", ["weight", "base"])
@pytest.mark.parametrize("k,m,T,n,r", [(200, 415, 10, 57, 88), (131, 64, 64, 3, 128), (66, 130, 33, 5, 17), (63, 65, 2, 9, 8)])
def test_few_tokens_of_many_ranks(ctx, dtype, shared, k, m, T, n, r):
    """Columns that fill no block of 64, ranks that fill no round of warps, adapters without a token."""
    L = draw(dtype, k, m, T, n, r, shared=shared, seed=6)
    check(run(ctx, L, dtype), L, dtype)


def test_a_weight_is_not_looked_at_where_its_gradient_is_not_wanted(ctx):
    from paper_2401_04044_b200 import Projection
    L = draw("bf16", 72, 88, 20, 3, 8)
    D = {k: None if v is None else v.cuda() for k, v in L.items()}
    W = torch.full((72 * 88 + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")[1:1 + 72 * 88].view(72, 88)      # on two bytes
    p, dA, dB = Projection(72, 88, torch.bfloat16), torch.empty_like(D["A"]), torch.empty_like(D["B"])
    ctx.ensure_workspace(ctx.adapter_workspace_size(p, 3, 8, 20))
    ctx.adapter_backward(p, D["X"], D["A"], D["B"], D["index"], D["dY"], W=W, base=D["X"], scale=D["scale"], dA=dA, dB=dB)
    ctx.poll()
    check({"dA": dA.cpu(), "dB": dB.cpu()}, L, "bf16")
