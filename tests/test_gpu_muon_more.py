"""More of the update by orthogonalised momentum, against the same iteration in 64 bits (tolerances: those of
test_gpu_muon.py, derived there, where nothing else is said)."""
import numpy as np
import pytest
import torch

from test_gpu_muon import DT, STANDARD, TOL, draw, near, orthogonal64, orthogonalize

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2401_04044_b200 import Context, build
    build.build()
    c = Context(0)
    c.ensure_workspace(1 << 20)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(64, 512), (4096, 64), (49, 2118), (8, 4100), (33, 4096)])
def test_few_thin_matrices_again_and_again(ctx, rows, cols, dtype):
    """Matrices whose parts the blocks of a cluster add up, many calls behind one another without a wait: each has the bits
    that it has in a list too long for clusters, where one block adds them up."""
    ms = [draw(rows, cols, DT[dtype], seed=s, noise=0.1 + 0.2 * s) for s in range(20)]
    many = orthogonalize(ctx, ms)
    ins, outs = [m.cuda() for m in ms], [torch.empty_like(m, device="cuda") for m in ms]
    lists = [ctx.orthogonal_list(ins[i:i + 2], outs[i:i + 2]) for i in range(0, 20, 2)]
    for _ in range(10):
        for o in outs:
            o.zero_()
        for lst in lists:
            ctx.orthogonalize(lst)
        ctx.poll()
        assert all(torch.equal(a, b) for a, b in zip(outs, many))
    near(many[3], orthogonal64(ms[3].double().numpy()), TOL[dtype])


@pytest.mark.parametrize("broken", [0, 1, 2, 4, 5, 200, 299])
def test_a_report_names_the_matrix_by_its_place_in_the_list(ctx, broken):
    """Thin and other matrices, several shapes, and more of them than one run takes."""
    from paper_2401_04044_b200 import FFSplitError
    shapes = [(300, 200), (16, 40), (130, 260), (300, 200), (40, 16), (70, 71)] + [(9, 11), (66, 67), (12, 8)] * 98
    g = [torch.randn(*s, device="cuda") for s in shapes]
    g[broken][-1, -1] = float("nan")
    lst = ctx.orthogonal_list(g, [torch.empty_like(t) for t in g])
    ctx.ensure_workspace(ctx.muon_workspace_size(lst))
    ctx.orthogonalize(lst)
    with pytest.raises(FFSplitError, match=rf"\(detail {broken}, ") as e:
        ctx.poll()
    assert e.value.code == 6
    ctx.poll()


@pytest.mark.parametrize("gdt,odt", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("shape", [(24, 100), (200, 90), (90, 1500), (640, 1000), (640, 700)])
def test_an_orthogonal_factor_of_momentum(ctx, shape, gdt, odt):
    """Without weights, with momentum that moves on: out = X of U, in either type."""
    from paper_2401_04044_b200 import MuonList
    g, m = draw(*shape, DT[gdt], seed=3).cuda(), 4 * draw(*shape, torch.float32, seed=4).cuda()
    out, moved = torch.empty(*shape, dtype=DT[odt], device="cuda"), torch.empty(*shape, device="cuda")
    lst = MuonList(0, [g], None, [m], out=[out], out_momenta=[moved])
    ctx.ensure_workspace(ctx.muon_workspace_size(lst))
    ctx.muon_step(lst, 0.5)
    ctx.poll()
    m64 = 0.5 * m.double() + g.double()
    near(moved, m64.cpu(), 2.0 ** -22)      # (two operations; near() asks for 8 times that of single elements)
    near(out, orthogonal64((g.double() + 0.5 * m64).cpu().numpy()), TOL[gdt] + (2.0 ** -8 if odt == "bf16" else 0.0))


@pytest.mark.parametrize("rows,cols", [(65, 1 << 18), (65, (1 << 18) + 8), ((1 << 20) + 1, 66), (65, 1 << 22), (520, 1 << 20)])
def test_long_sums(ctx, rows, cols):
    """The square's diagonal is a sum of as many terms of one sign as the longer side has, far more than a running sum in the tensor
    cores can take."""
    g = torch.Generator(device="cuda").manual_seed(9)
    m = torch.randn(rows, cols, generator=g, device="cuda").bfloat16()
    out = torch.empty_like(m)
    lst = ctx.orthogonal_list([m], [out])
    ctx.ensure_workspace(ctx.muon_workspace_size(lst))
    ctx.orthogonalize(lst)
    ctx.poll()
    x, o = (m, out) if rows <= cols else (m.t(), out.t())
    gram = torch.zeros(len(x), len(x), dtype=torch.float64, device="cuda")
    for at in range(0, x.shape[1], 1 << 18):
        piece = x[:, at:at + (1 << 18)].double()
        gram += piece @ piece.t()
    eye = torch.eye(len(x), dtype=torch.float64, device="cuda")
    norm = gram.trace().sqrt() + 1e-7
    s, Q = gram / norm ** 2, eye / norm
    for a, b, c in STANDARD:
        A = a * eye + b * s + c * (s @ s)
        Q, s = Q @ A, A @ s @ A
    for at in (0, x.shape[1] - 4096):
        near(o[:, at:at + 4096], (Q @ x[:, at:at + 4096].double()).cpu(), TOL["bf16"])


@pytest.mark.parametrize("kind", ["gauss", "positive"])
@pytest.mark.parametrize("rows,cols", [(65, 1024), (256, 1024), (512, 1024), (512, 4096), (4096, 512), (512, 1 << 15), (1024, 2752), (2048, 2048)])
def test_singular_values_close_together_in_fp32(ctx, rows, cols, kind):
    """1e-5 in fp32: S is summed in parts of 256 terms of one sign; a term loses half of 2^-24 of the running sum on average, which is
    half of the part's on average: 256 x 2^-26 = 3.8e-6 of S.  That enters through b s^2 + 2 c s^4, 0.71 where all singular
    values are near 1 and the result is 0.7: 3.8e-6, and as much again from the iterations before the last one.  Values that are
    close together do not average this out.  (P's own sums: parts of 64 terms.)"""
    g = torch.Generator().manual_seed(10)
    m = torch.randn(rows, cols, generator=g) if kind == "gauss" else torch.rand(rows, cols, generator=g)
    got, = orthogonalize(ctx, [m])
    near(got, orthogonal64(m.double().numpy()), TOL["f32"])


def test_a_list_of_several_runs(ctx):
    """More than the three gigabytes that are worked on at once, shapes in turn: every matrix has the bits that it has alone."""
    g = torch.Generator(device="cuda").manual_seed(12)
    shapes = [(3000, 9000), (9000, 3000), (40, 9000), (3000, 3100)] * 4
    ms = [torch.randn(*s, generator=g, device="cuda").bfloat16() for s in shapes]
    outs = [torch.empty_like(m) for m in ms]
    lst = ctx.orthogonal_list(ms, outs)
    each = sum(ctx.muon_workspace_size(ctx.orthogonal_list([m], [o])) - ctx.muon_workspace_size(ctx.orthogonal_list([], [])) for m, o in zip(ms, outs))
    assert ctx.muon_workspace_size(lst) <= 3.1e9 < each
    ctx.ensure_workspace(ctx.muon_workspace_size(lst))
    ctx.orthogonalize(lst)
    ctx.poll()
    for m, o in zip(ms, outs):
        alone = torch.empty_like(o)
        ctx.orthogonalize(ctx.orthogonal_list([m], [alone]))
        ctx.poll()
        assert torch.equal(alone, o)
