"""Host-only checks of the training calls: size queries and the refusals that need no GPU."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2401_04044_b200 import binding, build
    build.build()
    return binding.load_library()


def sizes(lib, d, m, act, dtype, T):
    from paper_2401_04044_b200 import binding as b
    saved, ws = C.c_size_t(), C.c_size_t()
    rc = lib.ffsplit_train_sizes(C.byref(b.Shape(d, m, act, dtype)), T, C.byref(saved), C.byref(ws))
    return rc, saved.value, ws.value


def test_sizes_follow_what_is_kept(lib):
    from paper_2401_04044_b200 import binding as b
    # per token and neuron: G and U in 20 bits and H in 16; Z in 20 and H in 16; fp32: 32 bits each and three planes of H
    for act, dtype, per in ((b.SWIGLU, b.BF16, 7.0), (b.GELU_ERF, b.BF16, 4.5), (b.SWIGLU, b.F32, 14.0), (b.GELU_TANH, b.F32, 10.0)):
        rc, saved, ws = sizes(lib, 1024, 2752, act, dtype, 2048)
        assert rc == 0 and 2048 * 2752 * per <= saved <= 2048 * 2816 * per + 1024
        assert ws >= 65536 + 2048 * 2752 * 2
    # more tokens never need less, from one token on
    last = (0, 0)
    for T in (1, 2, 31, 32, 33, 1000, 8192, 100000):
        rc, saved, ws = sizes(lib, 520, 771, b.GELU_ERF, b.BF16, T)
        assert rc == 0 and saved >= last[0] and ws >= last[1]
        last = (saved, ws)
    # either pointer may be left out
    assert lib.ffsplit_train_sizes(C.byref(b.Shape(64, 64, b.SWIGLU, b.BF16)), 4, None, None) == 0


def test_size_refusals(lib):
    from paper_2401_04044_b200 import binding as b
    assert sizes(lib, 60, 64, b.SWIGLU, b.BF16, 4)[0] == 2       # bf16: d a multiple of 8
    assert sizes(lib, 60, 64, b.SWIGLU, b.F32, 4)[0] == 0
    assert sizes(lib, 64, 0, b.SWIGLU, b.BF16, 4)[0] == 2
    assert sizes(lib, 64, 64, 9, b.BF16, 4)[0] == 1
    assert sizes(lib, 64, 64, b.SWIGLU, 7, 4)[0] == 4
    for T in (0, -1, 1 << 40):
        assert sizes(lib, 64, 64, b.SWIGLU, b.BF16, T)[0] == 2
    assert lib.ffsplit_train_sizes(None, 4, None, None) == 1
    n = C.c_size_t()
    assert lib.ffsplit_grad_workspace_size(-1, C.byref(n)) == 1 and lib.ffsplit_grad_workspace_size(3, None) == 1
    assert lib.ffsplit_grad_workspace_size(0, C.byref(n)) == 0 and n.value >= 65536
    few = n.value
    assert lib.ffsplit_grad_workspace_size(5000, C.byref(n)) == 0 and n.value > few


def test_calls_without_a_context_are_refused(lib):
    assert lib.ffsplit_train_forward(None, None, None, None, 1, None, 0, None, None) == 1
    assert lib.ffsplit_train_backward(None, None, None, None, 1, None, 0, None, None, None) == 1
    assert lib.ffsplit_grad_norm(None, None, 0, None, None) == 1
    assert lib.ffsplit_grad_clip(None, None, 0, 1.0, None, None) == 1


def test_gradient_list_checks_its_tensors():
    from paper_2401_04044_b200 import FFSplitError, GradList
    g = torch.ones(6)
    for grads, out, code in (([g], None, 1), ([g.half()], None, 4), ([g], [g.double()], 4), ([g], [], 2), ([g[::2]], None, 2)):
        with pytest.raises(FFSplitError) as e:
            GradList(0, grads, out)
        assert e.value.code == code
    empty = GradList(0, [])
    assert empty.count == 0 and C.sizeof(empty.array) >= 32


@pytest.fixture
def idle(monkeypatch):
    """A context over a library that is not there, and the list of what was done in order."""
    from paper_2401_04044_b200 import Context
    done, capturing = [], []

    class Library:
        def ffsplit_set_workspace(self, handle, ptr, nbytes):
            done.append("set")
            return 0

        def ffsplit_last_error(self, handle):
            return b""

    c = Context.__new__(Context)
    c.lib, c.h, c.device, c._ws = Library(), None, 0, None
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: done.append("wait"))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: bool(capturing))
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k).zero_())
    return c, done, capturing


def test_a_workspace_is_set_on_an_idle_device_and_not_in_a_capture(idle):
    from paper_2401_04044_b200 import FFSplitError
    c, done, capturing = idle
    memory = torch.zeros(1 << 17, dtype=torch.uint8)
    c.set_workspace(memory)
    assert done == ["wait", "set"] and c._ws is memory
    capturing.append(True)
    with pytest.raises(FFSplitError) as e:
        c.set_workspace(torch.zeros(1 << 18, dtype=torch.uint8))
    assert e.value.code == 1 and done == ["wait", "set"] and c._ws is memory


def test_a_growing_workspace_keeps_a_condition_that_was_not_reported(idle):
    c, done, _ = idle
    c.ensure_workspace(1 << 16)
    first = c._ws
    first[:12].view(torch.int32).copy_(torch.tensor([6, 77, 14], dtype=torch.int32))
    c.ensure_workspace(1 << 16)
    assert c._ws is first and done == ["wait", "set"]
    c.ensure_workspace(1 << 17)
    assert c._ws is not first and c._ws.numel() == 1 << 17 and done == ["wait", "set", "wait", "set", "wait"]
    assert c._ws[:12].view(torch.int32).tolist() == [6, 77, 14]


def test_a_workspace_that_a_graph_uses_stays_allocated(idle, monkeypatch):
    import weakref
    from paper_2401_04044_b200 import FFSplitError
    c, _, _ = idle
    capturing = []
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: bool(capturing))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    for name in ("ffsplit_grad_norm", "ffsplit_poll"):
        setattr(c.lib, name, lambda *a: 0)
    norm = lambda: c.lib.ffsplit_grad_norm(c.h, None, 0, None, c._stream(None))  # noqa: E731
    c.ensure_workspace(1 << 16)
    norm()
    unused = weakref.ref(c._ws)
    c.ensure_workspace(1 << 17)
    assert unused() is None
    capturing.append(True)
    norm()
    capturing.clear()
    used, where = weakref.ref(c._ws), c._ws.data_ptr()
    c.ensure_workspace(1 << 18)
    plain = weakref.ref(c._ws)
    c.ensure_workspace(1 << 19)
    assert used() is not None and used().data_ptr() == where and plain() is None
    # what a replay records there is reported as well, once
    used()[:12].view(torch.int32).copy_(torch.tensor([6, 5, 14], dtype=torch.int32))
    with pytest.raises(FFSplitError) as e:
        c.poll()
    assert e.value.code == 6
    c.poll()


def test_a_condition_that_moved_on_is_reported_once(idle, monkeypatch):
    c, _, _ = idle
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    c.lib.ffsplit_poll = lambda *a: 0      # (the library reports, and clears, what the new workspace holds)
    c.ensure_workspace(1 << 16)
    c._in_graph = True
    c._ws[:12].view(torch.int32).copy_(torch.tensor([6, 0, 14], dtype=torch.int32))
    c.ensure_workspace(1 << 17)
    assert len(c._retired) == 1 and c._ws[:12].view(torch.int32).tolist() == [6, 0, 14]
    c.poll()
