"""Tensors of more than 2^31 elements in the update of matrices and in the adapters: places that pass 32 bits.  Results are looked
at in 64 bits on the device, whole or, of the largest, in stretches from both ends and the middle.  Tolerances: those of
test_gpu_muon.py and test_gpu_adapter.py, derived there."""
import pytest
import torch

from test_gpu_adapter import DT, TOL as ADAPTER_TOL
from test_gpu_muon import STANDARD, TOL as MUON_TOL

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    from paper_2401_04044_b200 import Context, build
    build.build()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("100 GB of device memory are needed")
    c = Context(0)
    yield c
    c.close()
    torch.cuda.empty_cache()


def near(got, ref, tol):
    err, big = float((got.double() - ref).norm() / ref.norm()), float((got.double() - ref).abs().max() / ref.abs().max())
    assert err <= tol and big <= 8 * tol, (err, big)


@pytest.mark.parametrize("rows,cols", [(70, (1 << 25) + 5), ((1 << 25) + 5, 70), (33, (1 << 27) + 3), ((1 << 27) + 8, 24)])
def test_orthogonal_factor(ctx, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows % 97)
    p, tall = min(rows, cols), rows > cols
    mix = torch.randn(p, p, generator=g, device="cuda")
    m = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    long = m if tall else m.t()                     # [q, p], a stretch of q at a time
    step, q = 1 << 21, max(rows, cols)
    gram = torch.zeros(p, p, dtype=torch.float64, device="cuda")
    for at in range(0, q, step):
        piece = long[at:at + step]
        piece.copy_(torch.randn(piece.shape, generator=g, device="cuda") @ mix)
        x = piece.double()
        gram += x.t() @ x
    out = torch.full((rows * cols + 64,), -7.0, dtype=torch.bfloat16, device="cuda")
    o = out[32:32 + rows * cols].view(rows, cols)
    lst = ctx.orthogonal_list([m], [o])
    ctx.ensure_workspace(ctx.muon_workspace_size(lst))
    ctx.orthogonalize(lst)
    ctx.poll()
    assert (out[:32] == -7).all() and (out[-32:] == -7).all()
    # X_n = U Q with Q a polynomial in the Gram matrix
    norm = gram.trace().sqrt() + 1e-7
    s, Q = gram / norm ** 2, torch.eye(p, dtype=torch.float64, device="cuda") / norm
    for a, b, c in STANDARD:
        A = a * torch.eye(p, dtype=torch.float64, device="cuda") + b * s + c * (s @ s)
        Q, s = Q @ A, A @ s @ A
    result = o if tall else o.t()
    for at in (0, q // 2 - 500, (1 << 31) // p - 1000, q - 2000):
        near(result[at:at + 2000], long[at:at + 2000].double() @ Q, MUON_TOL["bf16"])


@pytest.mark.parametrize("shared", ["weight", "base"])
@pytest.mark.parametrize("k,m", [(72, 8192), (8192, 72), (72, 8191)])
def test_tokens(ctx, k, m, shared):
    from paper_2401_04044_b200 import Projection
    g, T, n, r, dt = torch.Generator(device="cuda").manual_seed(k), 263001, 3, 8, torch.bfloat16
    new = lambda s, *shape: torch.empty(*shape, dtype=dt, device="cuda").normal_(0.0, s, generator=g)  # noqa: E731
    X, dY, W, A, B = new(1.0, T, k), new(0.01, T, m), new(k ** -0.5, k, m), new(k ** -0.5, n, k, r), new(r ** -0.5, n, r, m)
    index = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    Y, dX, dA, dB = new(1.0, T, m), new(1.0, T, k), torch.empty_like(A), torch.empty_like(B)
    weight = shared == "weight"
    places = (0, T // 2, (1 << 31) // max(k, m) - 150, T - 300)
    before = {at: (Y[at:at + 300].double(), dX[at:at + 300].double()) for at in places}
    p = Projection(k, m, dt)
    ctx.ensure_workspace(ctx.adapter_workspace_size(p, n, r, T))
    ctx.adapter_forward(p, X, A, B, index, Y, W=W if weight else None, base=None if weight else Y)
    ctx.adapter_backward(p, X, A, B, index, dY, W=W if weight else None, base=None if weight else dX, dX=dX, dA=dA, dB=dB)
    ctx.poll()
    mine = [(index == i).double().unsqueeze(1) for i in range(n)]
    for at in places:
        s = slice(at, at + 300)
        x, d = X[s].double(), dY[s].double()
        y, z = (x @ W.double(), d @ W.double().t()) if weight else before[at]
        for i in range(n):
            y = y + mine[i][s] * (x @ A[i].double() @ B[i].double())
            z = z + mine[i][s] * (d @ B[i].double().t() @ A[i].double().t())
        near(Y[s], y, ADAPTER_TOL["bf16"])
        near(dX[s], z, ADAPTER_TOL["bf16"])
    refA, refB = torch.zeros(n, k, r, dtype=torch.float64, device="cuda"), torch.zeros(n, r, m, dtype=torch.float64, device="cuda")
    for at in range(0, T, 16384):
        s = slice(at, at + 16384)
        x, d = X[s].double(), dY[s].double()
        for i in range(n):
            refA[i] += x.t() @ (mine[i][s] * (d @ B[i].double().t()))
            refB[i] += (mine[i][s] * (x @ A[i].double())).t() @ d
    near(dA, refA, ADAPTER_TOL["bf16"])
    near(dB, refB, ADAPTER_TOL["bf16"])


@pytest.mark.parametrize("dtype,T", [("bf16", 20), ("bf16", 200), ("f32", 20), ("f32", 200)])
@pytest.mark.parametrize("k,m", [(8192, 64), (64, 8192)])
def test_factors(ctx, dtype, T, k, m):
    """5000 adapters of rank 64, the last ones among those that are used."""
    from paper_2401_04044_b200 import Projection
    g, n, r, dt = torch.Generator(device="cuda").manual_seed(T), 5000, 64, DT[dtype]
    new = lambda s, *shape: torch.empty(*shape, dtype=dt, device="cuda").normal_(0.0, s, generator=g)  # noqa: E731
    X, dY, A, B = new(1.0, T, k), new(0.01, T, m), new(k ** -0.5, n, k, r), new(r ** -0.5, n, r, m)
    index = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    index[:12] = torch.tensor([n - 1, n - 2, 4096, 4095, 0, n - 1, 4096, 4097, n - 1, 2, 0, -1], dtype=torch.int32)
    Y, dX, dA, dB = torch.empty(T, m, dtype=dt, device="cuda"), torch.empty(T, k, dtype=dt, device="cuda"), torch.empty_like(A), torch.empty_like(B)
    p = Projection(k, m, dt)
    ctx.ensure_workspace(ctx.adapter_workspace_size(p, n, r, T))
    dA.fill_(-7.0)
    dB.fill_(-7.0)
    ctx.adapter_forward(p, X, A, B, index, Y)
    ctx.adapter_backward(p, X, A, B, index, dY, dX=dX, dA=dA, dB=dB)
    ctx.poll()
    refY, refX = torch.zeros(T, m, dtype=torch.float64, device="cuda"), torch.zeros(T, k, dtype=torch.float64, device="cuda")
    used = sorted(set(index.tolist()) - {-1})
    for i in used:
        t = (index == i).nonzero().flatten()
        x, d, a, b = X[t].double(), dY[t].double(), A[i].double(), B[i].double()
        refY[t], refX[t] = x @ a @ b, d @ b.t() @ a.t()
        near(dA[i], x.t() @ (d @ b.t()), ADAPTER_TOL[dtype])
        near(dB[i], (x @ a).t() @ d, ADAPTER_TOL[dtype])
    near(Y, refY, ADAPTER_TOL[dtype])
    near(dX, refX, ADAPTER_TOL[dtype])
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[used] = False
    for v in (dA, dB):
        assert all(bool((v[at:at + 500][rest[at:at + 500]] == 0).all()) for at in range(0, n, 500))
