"""The optimiser for matrices without a GPU: what it does around the library's call, which is stood in for by one that changes
nothing."""
import pytest
import torch


class Library:
    """Stands in for a Context: takes tensors of the CPU and records the calls."""
    device = -1      # (what get_device() gives for them)

    def __init__(self):
        self.lists, self.size = [], 0      # of every call, and of the workspace

    def muon_workspace_size(self, tensors):
        return 100 * tensors.count

    def ensure_workspace(self, nbytes):
        self.size = max(self.size, nbytes)

    def muon_step(self, tensors, *args):
        assert 100 * tensors.count <= self.size
        self.lists.append(tensors)


def parameter(*shape):
    return torch.randn(*shape).requires_grad_()


def test_a_graph_from_before_a_step_is_refused():
    """A step writes to the parameters by their addresses; autograd has to know, or a graph that was kept gives gradients from
    the values after the step."""
    from paper_2401_04044_b200.train import Muon
    lib, W, stack, other = Library(), parameter(4, 6), parameter(2, 3, 5), parameter(4, 6)
    opt = Muon(lib, [W, stack, other])
    for p in (W, stack):
        kept = (p * p).sum()
        kept.backward(retain_graph=True)
        before = p._version
        opt.step()
        assert p._version > before and other._version == 0
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            kept.backward()
    (other * other).sum().backward()      # (no gradient until now: left as it was)
    assert len(lib.lists) == 2 and [t.count for t in lib.lists] == [1, 3]


def test_parameters_that_cannot_be_stepped_are_refused_when_they_are_added():
    from paper_2401_04044_b200 import FFSplitError
    from paper_2401_04044_b200.train import Muon
    bad = [torch.randn(6, 4).t().requires_grad_(), torch.randn(2, 5, 3).transpose(1, 2).requires_grad_(), torch.randn(0, 4).requires_grad_(),
           torch.randn(3, 0, 4).requires_grad_()]
    opt = Muon(Library(), [parameter(4, 6)])
    for p in bad:
        with pytest.raises(FFSplitError):
            Muon(Library(), [p])
        with pytest.raises(FFSplitError):
            opt.add_param_group({"params": [p]})
    assert len(opt.param_groups) == 1


def test_no_group_is_updated_where_a_later_one_cannot_be():
    from paper_2401_04044_b200.train import Muon
    lib, groups = Library(), [[parameter(4, 6)], [parameter(5, 7), parameter(2, 3, 4)], [parameter(9, 2)]]
    opt = Muon(lib, [{"params": g} for g in groups])
    for p in sum(groups, []):
        p.grad = torch.ones_like(p)
    opt.step()
    assert [t.count for t in lib.lists] == [1, 3, 1]
    for i, broken in ((1, torch.randn(7, 5).t()), (1, torch.randn(5, 7, dtype=torch.float64)), (2, torch.randn(2, 9).t())):
        p = groups[i][0]
        whole, p.grad = p.data, None
        p.data = broken
        p.grad = torch.ones(broken.shape, dtype=broken.dtype)
        with pytest.raises(RuntimeError):
            opt.step()
        assert len(lib.lists) == 3
        p.grad = None
        p.data = whole
        p.grad = torch.ones_like(p)
    opt.step()
    assert len(lib.lists) == 6


def test_a_matrix_that_is_named_twice_is_refused():
    """Two updates of one matrix in one call would run at the same time."""
    import warnings
    from paper_2401_04044_b200 import FFSplitError, MuonList
    from paper_2401_04044_b200.train import Muon
    g, w, m = (torch.randn(4, 6) for _ in range(3))
    other = [torch.randn(4, 6) for _ in range(4)]
    for kw in (dict(grads=[g, g], weights=[w, w]), dict(grads=[g, g], weights=[w, other[0]], momenta=[m, m]),
               dict(grads=[g, g], out=[w, w]), dict(grads=[g, g], weights=[w, other[0]], momenta=[m, other[1]], out=[other[2], other[3]], out_momenta=[m, other[3]])):
        with pytest.raises(FFSplitError) as e:
            MuonList(-1, **kw)
        assert e.value.code == 1
    # what is only read may be named again
    assert MuonList(-1, [g, g], [w, w], [m, m], out=other[:2], out_momenta=other[2:]).count == 2
    lib, p = Library(), parameter(4, 6)
    p.grad = torch.ones_like(p)
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")      # (torch's own, which is to become an error)
        opt = Muon(lib, [p, p])
    with pytest.raises(FFSplitError):
        opt.step()
    assert not lib.lists


def test_clipping_counts_as_a_change_of_the_gradients():
    from paper_2401_04044_b200.train import clip_grad_norm_

    class Clipping(Library):
        grad_workspace_size = staticmethod(lambda count: 0)

        def clip_grads(self, grads, max_norm, norm):
            self.lists.append(grads)

    lib, params, norm = Clipping(), [parameter(4, 6), parameter(3), parameter(2)], torch.zeros(1)
    for p in params[:2]:
        p.grad = torch.ones_like(p)
    x = torch.ones(4, 6, requires_grad=True)
    kept = (x * params[0].grad).sum()
    before = [p.grad._version for p in params[:2]]
    clip_grad_norm_(lib, params, 1.0, norm)
    assert len(lib.lists) == 1 and all(p.grad._version > v for p, v in zip(params, before))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.backward()


def test_an_unknown_optimiser_is_refused_and_a_rate_of_zero_is_taken(monkeypatch):
    from paper_2401_04044_b200 import train
    with pytest.raises(ValueError, match="adam"):
        train.finetune(None, 8, 16, optimizer="adam")
    rates = []

    def record(lib, d, m, act, *rest, **kw):
        rates.append(rest[-1])
        raise InterruptedError

    monkeypatch.setattr(train, "Context", lambda device: None)
    monkeypatch.setattr(train, "finetune", record)
    monkeypatch.setattr(train, "finetune_adapters", record)
    for argv in (["--lr", "0"], ["--lr", "0", "--optimizer", "muon"], ["--lr", "0", "--adapters", "4"], ["--lr", "0.5"], [], ["--optimizer", "muon"], ["--adapters", "4"]):
        with pytest.raises(InterruptedError):
            train.main(argv)
    assert rates == [0.0, 0.0, 0.0, 0.5, 5.0, 1e-3, 2e-2]
