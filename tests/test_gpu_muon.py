"""The update by orthogonalised momentum against the same iteration in 64 bits, on the same stored inputs.

Tolerances.  Momentum is two fp32 operations: 2^-23 of |beta M| + |G|.  The orthogonal factor, bf16 gradients: what is
rounded are the operands S and P = b S + c S^2 of each iteration's products, to fp16.  A rounding's rms is at most 0.58
2^-11 = 2.8e-4 of the value; where all singular values are near 1, which is the worst place, S enters the result with
b = 4.8 and P is 2.7 large while the result is 0.7: 1.9e-3 and 1.1e-3, 2.2e-3 together.  Iterations before the last one add
as much again at most (the map's slope there is about 1): 3.2e-3; with the rounding of a bf16 result, 1.7e-3, 3.6e-3.  6e-3
is asked for.  fp32 gradients carry 2^-22 instead of 2^-11: 1.6e-6 and as much from the sums; 1e-5 is asked for.  Single
elements are held to 8 times that bound of the largest element."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TOL = {"bf16": 6e-3, "f32": 1e-5}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
STANDARD = [(3.4445, -4.7750, 2.0315)] * 5


@pytest.fixture(scope="module")
def ctx():
    from paper_2401_04044_b200 import Context, build
    build.build()
    c = Context(0)
    c.ensure_workspace(1 << 20)
    yield c
    c.close()


def orthogonal64(u, coefficients=STANDARD):
    x = u / (np.linalg.norm(u) + 1e-7)
    x = x.T if u.shape[0] > u.shape[1] else x
    for a, b, c in coefficients:
        a, b, c = (float(np.float32(v)) for v in (a, b, c))
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def draw(rows, cols, dtype, seed=0, noise=0.3):
    g = torch.Generator().manual_seed(seed * 100003 + rows * 31 + cols)
    k = max(1, min(rows, cols) // 8)
    low = torch.randn(rows, k, generator=g) * torch.exp(-3 * torch.arange(k) / k) @ torch.randn(k, cols, generator=g)
    return (1e-3 * (low + noise * torch.randn(rows, cols, generator=g))).to(dtype)


def near(got, ref, tol, what=""):
    got, ref = got.double().cpu().numpy(), np.asarray(ref)
    norm, top = np.linalg.norm(ref), np.abs(ref).max()
    err, big = np.linalg.norm(got - ref), np.abs(got - ref).max()
    assert err <= tol * norm and big <= 8 * tol * top, f"{what}: {err / norm:.2e} of the norm, {big / top:.2e} of the largest element (<= {tol})"


def guarded(rows, cols, dtype, shift=0):
    """A matrix inside a buffer whose other elements must stay, `shift` elements off its alignment."""
    flat = torch.full((rows * cols + 64,), -7.0, dtype=dtype, device="cuda")
    return flat, flat[32 + shift:32 + shift + rows * cols].view(rows, cols)


def untouched(flat, t):
    at = t.storage_offset()
    return bool((flat[:at] == -7).all()) and bool((flat[at + t.numel():] == -7).all())


def orthogonalize(ctx, matrices, dtype=None, shift=0, **kw):
    ins = [m.cuda() for m in matrices]
    outs = [guarded(*m.shape, dtype or m.dtype, shift) for m in matrices]
    lst = ctx.orthogonal_list(ins, [t for _, t in outs])
    ctx.ensure_workspace(ctx.muon_workspace_size(lst))
    ctx.orthogonalize(lst, **kw)
    ctx.poll(kw.get("stream"))
    torch.cuda.synchronize()
    assert all(untouched(f, t) for f, t in outs), "written outside a matrix"
    return [t for _, t in outs]


SHAPES = [(1, 1), (1, 9), (9, 1), (2, 3), (5, 200), (300, 7), (16, 16), (16, 1024), (1000, 24), (31, 33), (32, 400), (33, 33),
          (40, 1111), (65, 64), (64, 256), (127, 700), (700, 127), (129, 130), (130, 129), (256, 256), (257, 515), (515, 257),
          (300, 1024), (1024, 300), (520, 521), (640, 2000)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonal_factor(ctx, rows, cols, dtype):
    m = draw(rows, cols, DT[dtype])
    got, = orthogonalize(ctx, [m])
    near(got, orthogonal64(m.double().numpy()), TOL[dtype])


@pytest.mark.parametrize("rows,cols", [(65, 65), (66, 1056), (66, 1057), (128, 2048), (193, 200), (255, 4080), (256, 257), (4096, 256), (1001, 250)])
@pytest.mark.parametrize("iterations", [1, 2, 5])
def test_small_squares(ctx, rows, cols, iterations):
    """Sides of at most 256, on both sides of q = 16 p, where the square and the polynomial of it are one launch."""
    m = draw(rows, cols, torch.bfloat16, seed=4)
    got, = orthogonalize(ctx, [m], coefficients=STANDARD[:iterations])
    near(got, orthogonal64(m.double().numpy(), STANDARD[:iterations]), TOL["bf16"])


def test_more_small_squares_than_pairs_of_multiprocessors(ctx):
    shapes = [(65, 90), (256, 300), (300, 256), (130, 129), (90, 65), (200, 200)]
    ms = [draw(*shapes[i % 6], torch.bfloat16, seed=i) for i in range(170)]
    for i, (m, o) in enumerate(zip(ms, orthogonalize(ctx, ms))):
        near(o, orthogonal64(m.double().numpy()), TOL["bf16"], f"matrix {i}")
        if i % 17 == 0:
            alone, = orthogonalize(ctx, [m])
            assert torch.equal(alone, o), f"matrix {i}"


@pytest.mark.parametrize("rows,cols,dtype", [(1500, 4100, "bf16"), (2900, 1100, "bf16"), (1100, 2000, "f32")])
def test_many_tiles(ctx, rows, cols, dtype):
    m = draw(rows, cols, DT[dtype], seed=1)
    got, = orthogonalize(ctx, [m])
    near(got, orthogonal64(m.double().numpy()), TOL[dtype])


@pytest.mark.parametrize("kind", ["rank one", "spread", "gauss", "small", "large", "largest"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(20, 90), (96, 300)])
def test_spectra(ctx, kind, dtype, rows, cols):
    """Few directions or very different ones: what is rounded off the large ones must not reach the others.

    X itself is rounded too, and that rounding has no direction: directions in which the matrix has (nearly) nothing are
    multiplied by a = 3.4445 in every iteration that is left.  X in 22 bits: 0.58 2^-22 |X| = 1.4e-7, of X0 (norm 1) times
    a^5 = 485, of the iterations after it a third, a ninth ... as much (together 1.41): 9.5e-5, next to a result of norm 0.7
    sqrt(rank) or more.  fp32 results are held to that on top (bf16: 22 bits too, below 2e-4 of 6e-3)."""
    g = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    p = min(rows, cols)
    m = {"rank one": lambda: r(rows, 1) @ r(1, cols),
         "spread": lambda: torch.linalg.qr(r(rows, p))[0] * torch.logspace(0, -3, p, dtype=torch.float64) @ torch.linalg.qr(r(cols, p))[0].T,
         "gauss": lambda: r(rows, cols), "small": lambda: 1e-12 * r(rows, cols), "large": lambda: 1e15 * r(rows, cols),
         "largest": lambda: 1e36 * r(rows, cols)}[kind]().to(DT[dtype])
    got, = orthogonalize(ctx, [m])
    ref = orthogonal64(m.double().numpy())
    near(got, ref, TOL[dtype] + 9.5e-5 / np.linalg.norm(ref))


@pytest.mark.parametrize("coefficients", [[(1.5, -0.5, 0.0)] * 3, [(1.0, 0.0, 0.0)], [(2.0, -1.5, 0.5)] * 16, [(1.875, -1.25, 0.375), (3.4445, -4.775, 2.0315)]])
def test_coefficients(ctx, coefficients):
    for shape in ((24, 100), (200, 90)):
        m = draw(*shape, torch.float32, seed=2)
        got, = orthogonalize(ctx, [m], coefficients=coefficients)
        near(got, orthogonal64(m.double().numpy(), coefficients), TOL["f32"])
        got, = orthogonalize(ctx, [m.bfloat16()], coefficients=coefficients)
        near(got, orthogonal64(m.bfloat16().double().numpy(), coefficients), TOL["bf16"])


def test_a_list_of_many_shapes_and_types(ctx):
    """Every matrix has the bits that it has alone, whatever else is in the list."""
    shapes = [(16, 40), (300, 200), (40, 16), (16, 40), (130, 260), (300, 200), (8, 8), (70, 71), (200, 300), (16, 40), (33, 500)]
    ms = [draw(r, c, torch.float32 if i % 3 == 1 else torch.bfloat16, seed=i) for i, (r, c) in enumerate(shapes)]
    got = orthogonalize(ctx, ms)
    for m, o in zip(ms, got):
        near(o, orthogonal64(m.double().numpy()), TOL["f32" if m.dtype is torch.float32 else "bf16"])
        alone, = orthogonalize(ctx, [m])
        assert torch.equal(alone, o)


def test_long_lists(ctx):
    ms = [draw(4 + i % 3, 6 + i % 5, torch.bfloat16, seed=i) for i in range(300)]
    for m, o in zip(ms, orthogonalize(ctx, ms)):
        near(o, orthogonal64(m.double().numpy()), TOL["bf16"])
    lst = ctx.orthogonal_list([], [])
    ctx.orthogonalize(lst)
    ctx.poll()


def step(ctx, shapes, gdt, wdt, beta=0.9, nesterov=True, in_place=False, shift=0, stepsize=0.05, decay=0.01, momentum=True, seed=0):
    G = [draw(r, c, DT[gdt], seed) for r, c in shapes]
    M = [draw(r, c, torch.float32, seed + 50) * 4 for r, c in shapes] if momentum else None
    W = [(0.02 * torch.randn(r, c, generator=torch.Generator().manual_seed(r + c))).to(DT[wdt]) for r, c in shapes]
    put = lambda t: guarded(*t.shape, t.dtype, shift)  # noqa: E731
    bufs = {"G": [put(t) for t in G], "W": [put(t) for t in W], "M": [put(t) for t in M] if momentum else None}
    for k, src in (("G", G), ("W", W), ("M", M)):
        for (_, d), s in zip(bufs[k] or [], src or []):
            d.copy_(s)
    out = bufs["W"] if in_place else [put(t) for t in W]
    out_m = bufs["M"] if in_place or not momentum else [put(t) for t in M]
    view = lambda b: None if b is None else [t for _, t in b]  # noqa: E731
    lst = ctx.muon_list(view(bufs["W"]), view(bufs["G"]), view(bufs["M"]), stepsize, decay, view(out), view(out_m))
    ctx.ensure_workspace(ctx.muon_workspace_size(lst))
    ctx.muon_step(lst, beta, nesterov)
    ctx.poll()
    torch.cuda.synchronize()
    for k in ("G", "W", "M"):
        for f, t in bufs[k] or []:
            assert untouched(f, t)
    for f, t in out + (out_m or []):
        assert untouched(f, t), "written outside a tensor"
    for i, (g, w) in enumerate(zip(G, W)):
        g64, w64 = g.double().numpy(), w.double().numpy()
        b64 = float(np.float32(beta))
        m64 = b64 * M[i].double().numpy() + g64 if momentum else g64
        u = (g64 + b64 * m64 if nesterov else m64) if momentum else g64
        if momentum:
            bound = 2.0 ** -23 * (np.abs(b64 * M[i].double().numpy()) + np.abs(g64))
            assert (np.abs(out_m[i][1].double().cpu().numpy() - m64) <= bound).all()
        o = orthogonal64(u)
        ref = (1 - float(np.float32(decay))) * w64 - float(np.float32(stepsize)) * o
        err = np.abs(out[i][1].double().cpu().numpy() - ref)
        # the factor's own error, the step in fp32, and the weight's rounding
        allowed = abs(stepsize) * 8 * TOL[gdt] * np.abs(o).max() + 2.0 ** -22 * np.abs(ref) + 2.0 ** -22 * np.abs(w64) + torch.finfo(DT[wdt]).eps / 2 * np.abs(ref)
        assert (err <= allowed).all(), f"matrix {i}: {err.max():.2e}, {(err / allowed).max():.2f} of what is allowed"
    return [t.clone() for t in view(out)]


@pytest.mark.parametrize("gdt,wdt", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("shapes", [[(16, 300)], [(300, 20), (260, 130), (17, 23)], [(128, 256)] * 3])
def test_step(ctx, shapes, gdt, wdt):
    step(ctx, shapes, gdt, wdt)


@pytest.mark.parametrize("shift", [1, 3, 8])
def test_tensors_off_16_bytes(ctx, shift):
    for shapes in ([(24, 64), (64, 136)], [(150, 56), (40, 330)]):
        step(ctx, shapes, "bf16", "bf16", shift=shift)
        step(ctx, shapes, "f32", "f32", shift=shift)


def test_in_place_and_forms_of_momentum(ctx):
    shapes = [(16, 80), (140, 300), (300, 140)]
    a = step(ctx, shapes, "bf16", "f32", in_place=True)
    b = step(ctx, shapes, "bf16", "f32", in_place=False)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    step(ctx, shapes, "f32", "f32", nesterov=False)
    step(ctx, shapes, "f32", "f32", beta=0.0)
    step(ctx, shapes, "bf16", "bf16", momentum=False)
    step(ctx, shapes, "f32", "f32", stepsize=0.0, decay=1.0)


def test_zeros(ctx):
    for shape in ((20, 50), (200, 150)):
        z = torch.zeros(*shape, dtype=torch.bfloat16)
        a, b = orthogonalize(ctx, [z, draw(*shape, torch.bfloat16)])
        assert (a == 0).all() and not (b == 0).all()


@pytest.mark.parametrize("shape", [(20, 50), (150, 220)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_gradient_that_is_not_finite_leaves_its_matrix_alone(ctx, shape, bad):
    from paper_2401_04044_b200 import FFSplitError
    G = [draw(*shape, torch.float32, seed=s).cuda() for s in range(3)]
    G[1][shape[0] // 2, shape[1] // 3] = bad
    W = [torch.randn(*shape, device="cuda") for _ in G]
    M = [torch.randn(*shape, device="cuda") for _ in G]
    before = [(w.clone(), m.clone()) for w, m in zip(W, M)]
    other = [torch.zeros_like(w) for w in W], [torch.zeros_like(m) for m in M]
    for out, out_m in ((None, None), other):
        lst = ctx.muon_list(W, G, M, 0.1, 0.1, out, out_m)
        ctx.ensure_workspace(ctx.muon_workspace_size(lst))
        ctx.muon_step(lst)
        with pytest.raises(FFSplitError) as e:
            ctx.poll()
        assert e.value.code == 6
        ctx.poll()
        w, m = (W, M) if out is None else (out, out_m)
        assert torch.equal(w[1], before[1][0]) and torch.equal(m[1], before[1][1])
        for i in (0, 2):
            assert torch.isfinite(w[i]).all() and torch.isfinite(m[i]).all() and not torch.equal(w[i], before[i][0])
        for i in range(3):
            W[i].copy_(before[i][0])
            M[i].copy_(before[i][1])
    out = [torch.zeros_like(g) for g in G]
    ctx.orthogonalize(ctx.orthogonal_list(G, out))
    with pytest.raises(FFSplitError):
        ctx.poll()
    assert torch.isnan(out[1]).all() and torch.isfinite(out[0]).all() and torch.isfinite(out[2]).all()


def test_refusals(ctx):
    from paper_2401_04044_b200 import FFSplitError
    a, b = torch.randn(8, 12, device="cuda"), torch.empty(8, 12, device="cuda")
    lst = ctx.orthogonal_list([a], [b])
    ctx.ensure_workspace(ctx.muon_workspace_size(lst))
    for kw in ({"coefficients": [(10.0, 0.0, 0.0)]}, {"coefficients": [(float("nan"), 0.0, 0.0)]}, {"iterations": 0}, {"iterations": 17},
               {"coefficients": [(100.0, -100.0, 0.9)]}, {"coefficients": []}, {"coefficients": [(1.0, 2.0)]}):
        with pytest.raises(FFSplitError) as e:
            ctx.orthogonalize(lst, **kw)
        assert e.value.code in (1, 2)
    with pytest.raises(FFSplitError):
        ctx.muon_step(ctx.muon_list([b], [a], None, float("inf"), 0.0))
    with pytest.raises(FFSplitError):
        ctx.muon_step(ctx.muon_list([b], [a], [torch.zeros_like(a)], 0.1, 0.0), beta=float("nan"))
    big = ctx.orthogonal_list([torch.empty(3000, 3000, device="cuda")], [torch.empty(3000, 3000, device="cuda")])
    small = torch.empty(1 << 17, dtype=torch.uint8, device="cuda")
    kept = ctx._ws
    ctx.set_workspace(small)
    with pytest.raises(FFSplitError) as e:
        ctx.orthogonalize(big)
    assert e.value.code == 5
    ctx.set_workspace(kept)


def test_other_stream_and_captured_replay(ctx):
    """A captured step that is replayed takes the gradients and momenta of each replay."""
    shapes = [(16, 120), (130, 200), (300, 140)]
    G = [draw(r, c, torch.bfloat16).cuda() for r, c in shapes]
    W = [torch.randn(r, c, device="cuda") for r, c in shapes]
    M = [torch.zeros(r, c, device="cuda") for r, c in shapes]
    state = [t.clone() for t in W + M]
    lst = ctx.muon_list(W, G, M, 0.02, 0.001)
    ctx.ensure_workspace(ctx.muon_workspace_size(lst))
    expected = []
    for i in range(3):
        ctx.muon_step(lst)
        expected.append([t.clone() for t in W + M])
    for t, s in zip(W + M, state):
        t.copy_(s)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx.muon_step(lst)
    stream.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(W + M, expected[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        ctx.muon_step(lst)
    for i in (1, 2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(W + M, expected[i]))
    ctx.poll()
