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
