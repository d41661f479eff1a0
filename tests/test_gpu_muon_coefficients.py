"""Iterations of one matrix with coefficients that differ from one to the next, against the same iteration in 64 bits.

Matrices of 512 rows and more, half as many columns again, take iterations in pairs (P2 P of two of them at once).
Tolerance: 6e-3 as derived in test_gpu_muon.py.  It holds for these lists a fortiori: what is rounded off S enters a result
p(s) with b s^2 / p(s), which is 4.8 / 0.7 for the standard triple and 1.5 or less for the others here, and a list that only
multiplies (b = c = 0) is off by the rounding of its result."""
import numpy as np
import pytest
import torch

from test_gpu_muon import TOL, draw, near, orthogonal64, orthogonalize

pytestmark = pytest.mark.gpu

MIXED = [(3.4445, -4.7750, 2.0315), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (1.5, -0.5, 0.0), (1.0, 0.25, -0.25)]
# every one of these is accepted alone, and so is the list; what two of them make of a pair is 256
STEEP = [(0.05, 0.0, 0.0), (0.05, 0.0, 0.0), (16.0, 0.0, 0.0), (16.0, 0.0, 0.0)]


@pytest.fixture(scope="module")
def ctx():
    from paper_2401_04044_b200 import Context, build
    build.build()
    c = Context(0)
    c.ensure_workspace(1 << 20)
    yield c
    c.close()


@pytest.mark.parametrize("shape", [(640, 2000), (2000, 640), (512, 768), (513, 771)])
@pytest.mark.parametrize("iterations", [1, 2, 3, 4, 5])
def test_pairs_of_different_triples(ctx, shape, iterations):
    m = draw(*shape, torch.bfloat16, seed=6)
    for triples in (MIXED[:iterations], MIXED[1:iterations + 1], MIXED[::-1][:iterations]):
        got, = orthogonalize(ctx, [m], coefficients=triples)
        near(got, orthogonal64(m.double().numpy(), triples), TOL["bf16"], triples)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(640, 2000), (2000, 640), (200, 90), (24, 100)])
@pytest.mark.parametrize("triples", [STEEP, [(1.0, 0.0, 0.0)] + STEEP, STEEP + MIXED[3:], [(0.05, 0.0, 0.0)] * 2 + [(15.0, 0.0, 0.0), (17.0, -40.0, 0.0)]])
def test_pairs_whose_product_is_large(ctx, shape, dtype, triples):
    m = draw(*shape, torch.float32 if dtype == "f32" else torch.bfloat16, seed=7)
    got, = orthogonalize(ctx, [m], coefficients=triples)
    near(got, orthogonal64(m.double().numpy(), triples), TOL[dtype], triples)


def test_lists_that_leave_next_to_nothing_before_an_iteration_are_refused(ctx):
    """1e-15 of the matrix is below what X is held with, and 64^8 of that is not: 0.28."""
    from paper_2401_04044_b200 import FFSplitError
    for shape in ((24, 100), (200, 90), (640, 2000)):
        m = draw(*shape, torch.bfloat16, seed=8)
        for triples in ([(1e-3, 0.0, 0.0)] * 5 + [(64.0, 0.0, 0.0)] * 8, [(0.9e-3, 0.0, 0.0), (64.0, 0.0, 0.0)]):
            with pytest.raises(FFSplitError) as e:
                orthogonalize(ctx, [m], coefficients=triples)
            assert e.value.code == 1
        # a list may end small, or with zeros
        for triples in ([(1e-3, 0.0, 0.0)], [(1.1e-3, 0.0, 0.0), (64.0, 0.0, 0.0)], [(0.0, 0.0, 0.0), (64.0, 0.0, 0.0)]):
            got, = orthogonalize(ctx, [m], coefficients=triples)
            ref = orthogonal64(m.double().numpy(), triples)
            if triples[0][0] == 0.0:
                assert (got == 0).all()
            else:
                near(got, ref, TOL["bf16"], triples)
