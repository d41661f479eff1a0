"""More of the update by orthogonalised momentum, against the same iteration in 64 bits (tolerances: those of
test_gpu_muon.py, derived there, where nothing else is said)."""
import numpy as np
import pytest
import torch

from test_gpu_muon import DT, TOL, draw, near, orthogonal64, orthogonalize

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
