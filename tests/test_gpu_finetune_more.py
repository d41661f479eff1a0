"""More of training with the optimiser and adapters."""
import pytest
import torch

from test_gpu_finetune import layer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2401_04044_b200 import Context, build
    build.build()
    c = Context(0)
    yield c
    c.close()


def test_graphs_that_hold_a_parameter_end_with_its_step(ctx):
    """Adapters beside a projection and a whole layer: a graph kept across a step is an error, a new one is not."""
    from paper_2401_04044_b200 import make_shape
    from paper_2401_04044_b200.train import Muon, adapted_ffn, ffn
    W, F, index, X, dY = layer("gelu_erf", 64, 136, 3, 8, 70, torch.bfloat16)
    shape, scale = make_shape(64, 136, "gelu_erf", torch.bfloat16), torch.ones(3, device="cuda")
    dense = [t.clone().requires_grad_() for t in (W["W1"], W["W2"])]
    factors = [t.requires_grad_() for v in F.values() for t in v]
    for params, run in ((factors, lambda: adapted_ffn(ctx, shape, X, W, F, index, scale)),
                        (dense, lambda: ffn(ctx, shape, X, *dense, W["b1"], W["b2"]))):
        opt = Muon(ctx, params)
        Y = run()
        Y.backward(dY, retain_graph=True)
        once = [p.grad.clone() for p in params]
        Y.backward(dY, retain_graph=True)      # (without a step between: the same again)
        assert all(torch.equal(p.grad, 2 * g) for p, g in zip(params, once))
        opt.step()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            Y.backward(dY)
        opt.zero_grad()
        run().backward(dY)
        assert all(torch.isfinite(p.grad).all() and not torch.equal(p.grad, g) for p, g in zip(params, once))
    ctx.poll()
