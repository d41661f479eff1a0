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
