"""Host-only checks of the calls for orthogonalised momentum and for adapters: size queries and refusals without a GPU."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2401_04044_b200 import binding, build
    build.build()
    return binding.load_library()


def muon_size(lib, shapes, count=None):
    from paper_2401_04044_b200 import binding as b
    array = (b.MuonTensor * max(1, len(shapes)))()
    for e, (rows, cols, g, w) in zip(array, shapes):
        e.rows, e.cols, e.grad_dtype, e.weight_dtype = rows, cols, g, w
    n = C.c_size_t()
    return lib.ffsplit_muon_workspace_size(C.byref(array), len(shapes) if count is None else count, C.byref(n)), n.value


def test_muon_sizes(lib):
    from paper_2401_04044_b200 import binding as b
    rc, none = muon_size(lib, [])
    assert rc == 0 and none >= 65536
    rc, one = muon_size(lib, [(256, 1024, b.BF16, b.BF16)])
    assert rc == 0 and one >= none + 256 * 1024 * 4
    assert muon_size(lib, [(1024, 256, b.BF16, b.F32)])[0] == 0
    # a long list is worked on in runs: its workspace does not grow without end
    few, many = muon_size(lib, [(4096, 11008, b.BF16, b.BF16)] * 4)[1], muon_size(lib, [(4096, 11008, b.BF16, b.BF16)] * 96)[1]
    assert few <= many <= 4 << 30
    assert muon_size(lib, [(0, 4, b.BF16, b.BF16)])[0] == 2 and muon_size(lib, [(4, -1, b.BF16, b.BF16)])[0] == 2
    assert muon_size(lib, [(1 << 20, 1 << 20, b.BF16, b.BF16)])[0] == 2 and muon_size(lib, [((1 << 31) - 1, 1, b.BF16, b.BF16)])[0] == 2
    assert muon_size(lib, [(4, 4, 7, b.BF16)])[0] == 4 and muon_size(lib, [(4, 4, b.F32, -1)])[0] == 4
    assert muon_size(lib, [], -1)[0] == 1
    assert lib.ffsplit_muon_workspace_size(None, 0, None) == 1 and lib.ffsplit_muon_workspace_size(None, 2, C.byref(C.c_size_t())) == 1


def test_adapter_sizes(lib):
    from paper_2401_04044_b200 import Projection
    size = lambda p, n, r, T: (lambda v: (lib.ffsplit_adapter_workspace_size(C.byref(p), n, r, T, C.byref(v)), v.value))(C.c_size_t())  # noqa: E731
    for dt in (torch.bfloat16, torch.float32):
        p, last = Projection(77, 131, dt), 0
        for T in (1, 2, 31, 256, 257, 5000):
            rc, n = size(p, 5, 16, T)
            assert rc == 0 and n >= max(last, 65536)
            last = n
        assert size(p, 5, 0, 4)[0] == 2 and size(p, 5, 129, 4)[0] == 2 and size(p, 0, 8, 4)[0] == 2 and size(p, 1 << 17, 8, 4)[0] == 2
        assert size(p, 1, 8, 0)[0] == 2 and size(p, 1, 8, 1 << 40)[0] == 2 and size(Projection(0, 8, dt), 1, 8, 1)[0] == 2
        assert size(Projection(8, -5, dt), 1, 8, 1)[0] == 2
    assert size(Projection(8, 8, 9), 1, 8, 1)[0] == 4
    assert lib.ffsplit_adapter_workspace_size(None, 1, 8, 1, C.byref(C.c_size_t())) == 1
    assert lib.ffsplit_adapter_workspace_size(C.byref(Projection(8, 8, 0)), 1, 8, 1, None) == 1


def test_calls_without_a_context_are_refused(lib):
    assert lib.ffsplit_muon_step(None, None, 0, 0.9, 1, None, 5, None) == 1
    assert lib.ffsplit_adapter_forward(None, None, None, None, None, None, None, 1, None, None) == 1
    assert lib.ffsplit_adapter_backward(None, None, None, None, None, None, 1, None, None, None) == 1


def test_muon_list_checks_its_tensors():
    from paper_2401_04044_b200 import FFSplitError, MuonList
    g = torch.ones(4, 6)
    cases = [(dict(grads=[g], weights=[g], momenta=[g]), 1), (dict(grads=[g], weights=[g.half()]), 4), (dict(grads=[g], weights=[g], out=[g.bfloat16()]), 4),
             (dict(grads=[g], weights=[g], momenta=[g.bfloat16()]), 4), (dict(grads=[g], weights=[]), 2), (dict(grads=[g]), 4),
             (dict(grads=[g[0]], weights=[g[0]]), 2), (dict(grads=[g], weights=[g.t()]), 2), (dict(grads=[g.t()], weights=[g.t()]), 2),
             (dict(grads=[g], weights=[g], out_momenta=[g]), 1), (dict(grads=[g], weights=[g], step=[1.0, 2.0]), 2)]
    for kw, code in cases:
        with pytest.raises(FFSplitError) as e:
            MuonList(0, **kw)
        assert e.value.code == code, kw
    assert MuonList(0, []).count == 0


def test_the_optimiser_checks_later_groups_and_loads_its_momentum_in_32_bits():
    from paper_2401_04044_b200 import FFSplitError
    from paper_2401_04044_b200.train import Muon
    params = lambda: [torch.ones(3, 5, dtype=torch.bfloat16, requires_grad=True), torch.ones(2, 4, 6, requires_grad=True)]  # noqa: E731
    first, second = params(), params()
    a, b = Muon(None, first[:1]), Muon(None, second[:1], lr=1.0)
    for opt, p in ((a, first[1]), (b, second[1])):
        opt.add_param_group({"params": [p], "lr": 0.5})
        for bad in (torch.ones(4, requires_grad=True), torch.ones(4, 4, dtype=torch.float16, requires_grad=True)):
            with pytest.raises(FFSplitError):
                opt.add_param_group({"params": [bad]})
        assert len(opt.param_groups) == 2
    for p in first:
        a.state[p]["momentum"] = torch.randn(p.shape)
    b.load_state_dict(a.state_dict())
    assert b.param_groups[0]["lr"] == 0.02
    for p, q in zip(first, second):
        m, n = a.state[p]["momentum"], b.state[q]["momentum"]
        assert n.dtype is torch.float32 and torch.equal(m, n) and m.data_ptr() != n.data_ptr()
