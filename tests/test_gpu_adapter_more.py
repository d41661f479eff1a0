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
