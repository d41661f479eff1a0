"""More of the adapters and their gradients, against plain implementations in 64 bits (inputs, tolerances and the reference:
those of test_gpu_adapter.py)."""
import numpy as np
import pytest
import torch

from test_gpu_adapter import DT, TOL, check, draw, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2401_04044_b200 import Context, build
    build.build()
    c = Context(0)
    c.ensure_workspace(1 << 20)
    yield c
    c.close()


@pytest.mark.parametrize("dtype,k,m,T,n,r", [("bf16", 256, 4096, 400, 5, 24), ("bf16", 4096, 256, 400, 5, 24), ("bf16", 1500, 200, 130, 1, 70),
                                             ("f32", 256, 4096, 400, 5, 24), ("bf16", 256, 4096, 40, 5, 24), ("bf16", 8200, 264, 4200, 3, 16)])
def test_a_gradient_has_the_same_bits_whichever_others_are_asked_for(ctx, dtype, k, m, T, n, r):
    """Sides of different length: each factor's product is cut into ranges by its own sizes."""
    L = draw(dtype, k, m, T, n, r, order="segments", seed=16)
    whole = run(ctx, L, dtype)
    check(whole, L, dtype)
    for want in (("dX",), ("dA",), ("dB",), ("dA", "dB"), ("dX", "dB"), ("dX", "dA")):
        for o, v in run(ctx, L, dtype, want=want).items():
            assert torch.equal(v, whole[o]), (want, o)


@pytest.mark.parametrize("shared,dtype,k,m,T,n", [(s, *c) for s in ("weight", "base", "alone")
                                                  for c in (("bf16", 72, 136, 20, 3), ("bf16", 72, 136, 90, 3), ("f32", 72, 136, 90, 3), ("bf16", 264, 8200, 4200, 3))
                                                  if (s, c[0]) != ("weight", "f32")])
@pytest.mark.parametrize("r", [1, 24])
def test_an_infinity_stays_one_where_the_formula_has_one(ctx, shared, dtype, k, m, T, n, r):
    """(An fp32 layer beside W is left out: its operands are sums of three terms, some of them negative or zero.)  Ranks are filled up to whole matrix instructions; an infinity times what they are filled with is not to be met.  Every
    factor is positive, so an infinite token makes every element of its row (and of the gradients it reaches) infinite."""
    L = draw(dtype, k, m, T, n, r, order="mixed", shared=shared, seed=17, bias=False, scaled=False)
    for o in ("A", "B", "W"):
        if L[o] is not None:
            L[o] = L[o].abs() + 2.0 ** -10
    clean = run(ctx, L, dtype)
    t = int(np.nonzero(L["index"].numpy() == 1)[0][0])
    rows = [i for i in range(T) if i != t]
    L["X"][t, 3], L["dY"][t, 5] = float("inf"), float("inf")
    got = run(ctx, L, dtype, want=("Y", "dX"))
    for o in ("Y", "dX"):
        assert torch.isposinf(got[o][t]).all(), o
        assert torch.equal(got[o][rows], clean[o][rows]), o


# (products with an extension, cut along K, with copies of ragged operands, on the CUDA cores, without a sort)
CHAIN = [("bf16", 264, 8200, 4200, 4, 16, "weight"), ("bf16", 8200, 264, 4201, 3, 72, "weight"), ("bf16", 4096, 264, 200, 5, 24, "weight"),
         ("bf16", 333, 1001, 300, 7, 12, "weight"), ("bf16", 712, 904, 777, 6, 40, "base"), ("f32", 1024, 520, 150, 4, 12, "weight"),
         ("f32", 100, 60, 30, 3, 8, "base"), ("bf16", 2048, 264, 33, 9, 16, "weight"), ("bf16", 70, 480008, 72, 2, 8, "weight")]


class Calls:
    """Buffers of a forward and a backward call; `inputs` are copied in on the stream, outputs are cloned on it."""

    def __init__(self, ctx, L, dtype):
        from paper_2401_04044_b200 import Projection
        self.ctx, self.D = ctx, {k: None if v is None else v.cuda().clone() for k, v in L.items()}
        (T, k), (n, _, r), m = L["X"].shape, L["A"].shape, L["B"].shape[2]
        self.p = Projection(k, m, DT[dtype])
        self.size = ctx.adapter_workspace_size(self.p, n, r, T)
        self.out = {o: torch.empty(s, dtype=DT[dtype], device="cuda") for o, s in (("Y", (T, m)), ("dX", (T, k)), ("dA", (n, k, r)), ("dB", (n, r, m)))}

    def load(self, L):
        for k, v in L.items():
            if v is not None:
                self.D[k].copy_(v, non_blocking=True)

    def __call__(self):
        D, o = self.D, self.out
        self.ctx.adapter_forward(self.p, D["X"], D["A"], D["B"], D["index"], o["Y"], W=D["W"], b=D["b"], base=D["base"], scale=D["scale"])
        self.ctx.adapter_backward(self.p, D["X"], D["A"], D["B"], D["index"], D["dY"], W=D["W"], base=D["base_dX"], scale=D["scale"], dX=o["dX"], dA=o["dA"], dB=o["dB"])

    def results(self):
        return {k: v.clone() for k, v in self.out.items()}


def equal(a, b):
    return all(torch.equal(a[k], b[k]) for k in a)


def test_calls_behind_one_another_without_a_wait(ctx):
    """All of these share one workspace, with new inputs from call to call and nothing between them but their kernels' own
    waits: each result has the bits of a call alone."""
    draws = [[{k: None if v is None else v.cuda() for k, v in draw(d, k, m, T, n, r, shared=s, order="mixed" if i else "segments", seed=30 + i).items()} for i in range(3)]
             for d, k, m, T, n, r, s in CHAIN]
    calls = [Calls(ctx, three[0], c[0]) for three, c in zip(draws, CHAIN)]
    ctx.ensure_workspace(max(c.size for c in calls))
    alone = []
    for c, three in zip(calls, draws):
        alone.append([])
        for L in three:
            c.load(L)
            torch.cuda.synchronize()
            c()
            ctx.poll()
            alone[-1].append(c.results())
    for c, three, results in zip(CHAIN, draws, alone):
        check({k: v.cpu() for k, v in results[1].items()}, {k: None if v is None else v.cpu() for k, v in three[1].items()}, c[0])
    for _ in range(3):
        got = []
        for i in range(3):
            for c, three in zip(calls, draws):
                c.load(three[i])
                c()
                c()
                got.append(c.results())
        ctx.poll()
        for i in range(3):
            for j in range(len(calls)):
                assert equal(got[i * len(calls) + j], alone[j][i]), (CHAIN[j], i)


@pytest.mark.parametrize("case", CHAIN[:7], ids=str)
def test_captured_and_replayed(ctx, case):
    """The same with a captured forward and backward of batches that are sorted, replayed with other inputs."""
    d, k, m, T, n, r, s = case
    Ls = [draw(d, k, m, T, n, r, shared=s, order="mixed", seed=40 + i) for i in range(3)]
    c = Calls(ctx, Ls[0], d)
    ctx.ensure_workspace(c.size)
    expected = []
    for L in Ls:
        c.load(L)
        c()
        ctx.poll()
        expected.append(c.results())
    check({k: v.cpu() for k, v in expected[2].items()}, Ls[2], d)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        c()
    for i in (2, 0, 1):
        c.load(Ls[i])
        for v in c.out.values():
            v.zero_()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert equal(c.out, expected[i]), i
    ctx.poll()


@pytest.mark.parametrize("dtype,T", [("bf16", 5), ("bf16", 300), ("f32", 70)])
@pytest.mark.parametrize("act", ["gelu_erf", "swiglu"])
def test_beside_a_split_layer(ctx, act, dtype, T):
    """A packed layer whose light neurons are factors gives what the adapters of its requests are added to, in place: a run of
    both, forward and the adapters' gradients."""
    from paper_2401_04044_b200 import Projection, make_shape
    d, m, k, r, n, rank = 136, 264, 40, 8, 5, 16
    g, dt = torch.Generator().manual_seed(T), DT[dtype]
    new = lambda s, *shape: (torch.randn(*shape, generator=g) * s).to(dt).cuda()  # noqa: E731
    gated = act == "swiglu"
    W1, W1u, W2 = new(d ** -0.5, d, m), new(d ** -0.5, d, m) if gated else None, new(m ** -0.5, m, d)
    b1, b2 = (None, None) if gated else (new(0.1, m), new(0.1, d))
    rows = m - k
    factors = {"A1": new(d ** -0.5, d, r), "B1": new(r ** -0.5, r, rows), "A2": new(rows ** -0.5, rows, r), "B2": new(r ** -0.5, r, d)}
    if gated:
        factors.update(A1u=new(d ** -0.5, d, r), B1u=new(r ** -0.5, r, rows))
    heavy = torch.randperm(m, generator=g)[:k].sort().values.to(torch.int32).cuda()
    shape = make_shape(d, m, act, dt)
    p = Projection(d, d, dt)
    ctx.ensure_workspace(max(ctx.workspace_size(shape, T, T, k, r), ctx.adapter_workspace_size(p, n, rank, T)))
    blob = torch.empty(ctx.pack_size(shape, k, r)[0], dtype=torch.uint8, device="cuda")
    ctx.pack(shape, W1, b1, W2, b2, heavy, k, factors, blob, W1u=W1u)
    L = draw(dtype, d, d, T, n, rank, shared="base", order="mixed", seed=50)
    L["base_dX"] = None
    D = {q: None if v is None else v.cuda() for q, v in L.items()}
    alone, Y = torch.empty(T, d, dtype=dt, device="cuda"), torch.empty(T, d, dtype=dt, device="cuda")
    ctx.forward(blob, D["X"], alone)
    ctx.poll()
    dX, dA, dB = torch.empty_like(D["X"]), torch.empty_like(D["A"]), torch.empty_like(D["B"])
    for _ in range(3):
        ctx.forward(blob, D["X"], Y)
        ctx.adapter_forward(p, D["X"], D["A"], D["B"], D["index"], Y, base=Y, scale=D["scale"])
        ctx.adapter_backward(p, D["X"], D["A"], D["B"], D["index"], D["dY"], scale=D["scale"], dX=dX, dA=dA, dB=dB)
    ctx.poll()
    ctx.blob_close(blob)
    # the layer's own output is what test_gpu_parity.py looks at; here it is the base, as it came
    L["base"] = alone.cpu()
    check({"Y": Y.cpu(), "dX": dX.cpu(), "dA": dA.cpu(), "dB": dB.cpu()}, L, dtype)


@pytest.mark.parametrize("T,n,k,m,r", [((1 << 18) + 1, 1, 72, 64, 8), ((1 << 20) + 3, 1, 64, 72, 72), ((1 << 20) + 129, 3, 136, 64, 20), ((1 << 19) + 64, 2, 33, 130, 128)])
def test_gradients_of_an_adapter_with_many_tokens(ctx, T, n, k, m, r):
    """All terms have one sign: a running sum in the tensor cores, which cut what they add, would lose 6e-3 of 2^20 terms.  (The
    tolerance is that of the other gradients: the parts' sums are in fp32.)"""
    from paper_2401_04044_b200 import Projection
    g = torch.Generator(device="cuda").manual_seed(T % 1000)
    new = lambda s, *shape: ((torch.rand(*shape, generator=g, device="cuda") + 0.5) * s).bfloat16()  # noqa: E731
    X, dY, A, B = new(1.0, T, k), new(1e-3, T, m), new(1.0 / k, n, k, r), new(1.0 / r, n, r, m)
    index = torch.zeros(T, dtype=torch.int32, device="cuda")      # (nearly all of the first one's: not in one run where there are others)
    index[5::1009] = n - 1
    index[7::997] = -1
    p, dA, dB = Projection(k, m, torch.bfloat16), torch.empty_like(A), torch.empty_like(B)
    ctx.ensure_workspace(ctx.adapter_workspace_size(p, n, r, T))
    ctx.adapter_backward(p, X, A, B, index, dY, dA=dA, dB=dB)
    ctx.poll()
    for i in range(n):
        t = (index == i).nonzero().flatten()
        x, d = X[t].double(), dY[t].double()
        for got, ref in ((dA[i], x.t() @ (d @ B[i].double().t())), (dB[i], (x @ A[i].double()).t() @ d)):
            err, big = float((got.double() - ref).norm()), float((got.double() - ref).abs().max())
            assert err <= TOL["bf16"] * float(ref.norm()) and big <= 8 * TOL["bf16"] * float(ref.abs().max()), (i, err / float(ref.norm()))
