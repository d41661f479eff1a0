"""ctypes binding of libffsplit (include/ffsplit.h).

Argument marshalling only: every step of the path (scoring, selection, packing,
forward) runs in the library's CUDA kernels.  torch is used for device memory
and streams.  There is no CPU fallback: loading fails loudly when the shared
library has not been built, and every call raises on a non-zero status.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libffsplit.so")

OK = 0
ERR_NAMES = {
    1: "INVALID_ARG", 2: "SHAPE", 3: "ALIGN", 4: "DTYPE", 5: "BUFFER_TOO_SMALL", 6: "NONFINITE",
    7: "BAD_BLOB", 8: "ARCH", 9: "CUDA", 10: "TIMEOUT", 11: "BAD_INDEX",
}
F32, BF16 = 0, 1
GELU_ERF, GELU_TANH, SWIGLU = 0, 1, 2
SCORE_EQ3, SCORE_ACT_ONLY, SCORE_SUM_NORM = 0, 1, 2
ACT_IDS = {"gelu_erf": GELU_ERF, "gelu_tanh": GELU_TANH, "swiglu": SWIGLU}
DTYPE_IDS = {torch.float32: F32, torch.bfloat16: BF16}
DTYPES = {F32: torch.float32, BF16: torch.bfloat16}
SCORE_IDS = {"eq3": SCORE_EQ3, "act_only": SCORE_ACT_ONLY, "sum_norm": SCORE_SUM_NORM}

EXPORTS = [
    "ffsplit_create", "ffsplit_destroy", "ffsplit_workspace_size", "ffsplit_set_workspace", "ffsplit_score",
    "ffsplit_select", "ffsplit_pack_size", "ffsplit_pack", "ffsplit_blob_open", "ffsplit_blob_section",
    "ffsplit_forward", "ffsplit_forward_host", "ffsplit_poll", "ffsplit_launch_count", "ffsplit_last_error",
    "ffsplit_version", "ffsplit_profile_begin", "ffsplit_profile_end", "ffsplit_forward_noalloc",
    "ffsplit_forward_dense", "ffsplit_score_activations", "ffsplit_score_host", "ffsplit_score_finalize",
    "ffsplit_blob_close", "ffsplit_stack_workspace_size", "ffsplit_forward_stack", "ffsplit_forward_stack_host",
    "ffsplit_debug_wait_timeout", "ffsplit_quant_pack_size", "ffsplit_quant_workspace_size", "ffsplit_quant_pack",
    "ffsplit_quant_blob_open", "ffsplit_quant_unpack", "ffsplit_quant_forward",
    "ffsplit_factor_workspace_size", "ffsplit_factor_light", "ffsplit_encoder_workspace_size", "ffsplit_encoder_forward",
    "ffsplit_train_sizes", "ffsplit_train_forward", "ffsplit_train_backward",
    "ffsplit_grad_workspace_size", "ffsplit_grad_norm", "ffsplit_grad_clip",
    "ffsplit_muon_workspace_size", "ffsplit_muon_step",
    "ffsplit_adapter_workspace_size", "ffsplit_adapter_forward", "ffsplit_adapter_backward",
]


class EncoderLayer(C.Structure):
    _fields_ = [("batch", C.c_int32), ("seq", C.c_int32), ("heads", C.c_int32), ("Wqkv_t", C.c_void_p), ("bqkv", C.c_void_p),
                ("Wo_t", C.c_void_p), ("bo", C.c_void_p), ("ln1_gamma", C.c_void_p), ("ln1_beta", C.c_void_p),
                ("ln2_gamma", C.c_void_p), ("ln2_beta", C.c_void_p), ("ln_eps", C.c_float), ("ffn_blob", C.c_void_p)]


class Shape(C.Structure):
    _fields_ = [("d", C.c_int32), ("m", C.c_int32), ("act", C.c_int32), ("dtype", C.c_int32)]


class Weights(C.Structure):
    _fields_ = [("W1", C.c_void_p), ("W1u", C.c_void_p), ("b1", C.c_void_p), ("W2", C.c_void_p), ("b2", C.c_void_p)]


class Factors(C.Structure):
    _fields_ = [("A1", C.c_void_p), ("B1", C.c_void_p), ("A1u", C.c_void_p), ("B1u", C.c_void_p),
                ("A2", C.c_void_p), ("B2", C.c_void_p), ("r", C.c_int32)]


class TrainGrads(C.Structure):
    _fields_ = [("dX", C.c_void_p), ("dW1", C.c_void_p), ("dW1u", C.c_void_p), ("db1", C.c_void_p), ("dW2", C.c_void_p),
                ("db2", C.c_void_p)]


class MuonTensor(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("momentum", C.c_void_p), ("momentum_out", C.c_void_p), ("weight", C.c_void_p),
                ("out", C.c_void_p), ("rows", C.c_int32), ("cols", C.c_int32), ("grad_dtype", C.c_int32),
                ("weight_dtype", C.c_int32), ("step", C.c_float), ("decay", C.c_float)]


class Projection(C.Structure):
    """A shared projection [inner, outer] and the type of its tensors."""
    _fields_ = [("inner", C.c_int32), ("outer", C.c_int32), ("dtype", C.c_int32)]

    def __init__(self, inner: int, outer: int, dtype):
        super().__init__(inner, outer, DTYPE_IDS[dtype] if isinstance(dtype, torch.dtype) else int(dtype))


class Adapters(C.Structure):
    _fields_ = [("A", C.c_void_p), ("B", C.c_void_p), ("scale", C.c_void_p), ("index", C.c_void_p), ("n", C.c_int32),
                ("r", C.c_int32)]


class AdapterGrads(C.Structure):
    _fields_ = [("dX", C.c_void_p), ("dA", C.c_void_p), ("dB", C.c_void_p)]


class FFSplitError(RuntimeError):
    def __init__(self, code: int, where: str, text: str = ""):
        self.code = code
        super().__init__(f"{where}: FFSPLIT_ERR_{ERR_NAMES.get(code, code)} {text}".strip())


_lib = None


def load_library(path: Optional[str] = None) -> C.CDLL:
    """Load libffsplit.so (built in-tree by paper_2401_04044_b200.build).  Raises if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise FileNotFoundError(
            f"{p} not found: build it with `python -m paper_2401_04044_b200.build` (there is no fallback path)")
    lib = C.CDLL(p)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    P = C.POINTER
    lib.ffsplit_create.argtypes = [P(vp), C.c_int]
    lib.ffsplit_destroy.argtypes = [vp]
    lib.ffsplit_workspace_size.argtypes = [P(Shape), i64, i64, i32, i32, P(sz)]
    lib.ffsplit_set_workspace.argtypes = [vp, vp, sz]
    lib.ffsplit_score.argtypes = [vp, P(Shape), P(Weights), vp, i64, i32, i32, vp, vp, vp]
    lib.ffsplit_select.argtypes = [vp, vp, i32, i32, vp, vp, vp]
    lib.ffsplit_pack_size.argtypes = [P(Shape), i32, i32, P(sz), P(sz)]
    lib.ffsplit_pack.argtypes = [vp, P(Shape), P(Weights), vp, i32, P(Factors), vp, sz, vp]
    lib.ffsplit_blob_open.argtypes = [vp, vp, sz, vp]
    lib.ffsplit_blob_close.argtypes = [vp, vp]
    lib.ffsplit_score_host.argtypes = [vp, P(Shape), P(Weights), vp, i64, i32, i32, vp, vp, vp]
    lib.ffsplit_score_finalize.argtypes = [vp, P(Shape), vp, i32, vp, vp, vp]
    lib.ffsplit_score_activations.argtypes = [vp, P(Shape), vp, i64, vp, i32, i32, vp, vp, vp]
    lib.ffsplit_forward_dense.argtypes = [vp, P(Shape), P(Weights), vp, i64, vp, vp]
    lib.ffsplit_stack_workspace_size.argtypes = [vp, P(vp), i32, i64, P(sz)]
    lib.ffsplit_forward_stack.argtypes = [vp, P(vp), i32, vp, i64, vp, vp]
    lib.ffsplit_forward_stack_host.argtypes = [vp, P(vp), i32, vp, i64, vp, vp]
    lib.ffsplit_debug_wait_timeout.argtypes = [vp, i64, vp]
    lib.ffsplit_quant_pack_size.argtypes = [P(Shape), i32, P(sz), P(sz)]
    lib.ffsplit_quant_workspace_size.argtypes = [P(Shape), i32, P(sz)]
    lib.ffsplit_quant_pack.argtypes = [vp, P(Shape), P(Weights), vp, i32, vp, vp, sz, vp]
    lib.ffsplit_quant_blob_open.argtypes = [vp, vp, sz, vp]
    lib.ffsplit_quant_unpack.argtypes = [vp, vp, i32, vp, vp, vp, vp]
    lib.ffsplit_quant_forward.argtypes = [vp, vp, vp, i64, vp, vp]
    lib.ffsplit_encoder_workspace_size.argtypes = [vp, vp, P(sz)]
    lib.ffsplit_encoder_forward.argtypes = [vp, vp, vp, vp, vp]
    lib.ffsplit_factor_workspace_size.argtypes = [vp, i32, i32, P(sz)]
    lib.ffsplit_factor_light.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.ffsplit_blob_section.argtypes = [vp, vp, i32, P(sz), P(i64), P(i64), P(i64)]
    lib.ffsplit_forward.argtypes = [vp, vp, vp, i64, vp, vp]
    lib.ffsplit_forward_host.argtypes = [vp, vp, vp, i64, vp, vp]
    lib.ffsplit_forward_noalloc.argtypes = [vp, vp, vp, i64, vp, vp]
    lib.ffsplit_train_sizes.argtypes = [P(Shape), i64, P(sz), P(sz)]
    lib.ffsplit_train_forward.argtypes = [vp, P(Shape), P(Weights), vp, i64, vp, sz, vp, vp]
    lib.ffsplit_train_backward.argtypes = [vp, P(Shape), P(Weights), vp, i64, vp, sz, vp, P(TrainGrads), vp]
    lib.ffsplit_grad_workspace_size.argtypes = [i32, P(sz)]
    lib.ffsplit_grad_norm.argtypes = [vp, vp, i32, vp, vp]
    lib.ffsplit_grad_clip.argtypes = [vp, vp, i32, C.c_float, vp, vp]
    lib.ffsplit_muon_workspace_size.argtypes = [vp, i32, P(sz)]
    lib.ffsplit_muon_step.argtypes = [vp, vp, i32, C.c_float, i32, vp, i32, vp]
    lib.ffsplit_adapter_workspace_size.argtypes = [P(Projection), i32, i32, i64, P(sz)]
    lib.ffsplit_adapter_forward.argtypes = [vp, P(Projection), vp, vp, vp, P(Adapters), vp, i64, vp, vp]
    lib.ffsplit_adapter_backward.argtypes = [vp, P(Projection), vp, vp, P(Adapters), vp, i64, vp, P(AdapterGrads), vp]
    lib.ffsplit_poll.argtypes = [vp, vp]
    lib.ffsplit_profile_begin.argtypes = [vp]
    lib.ffsplit_profile_end.argtypes = [vp, vp, i32, P(i32), P(C.c_double), P(C.c_double)]
    lib.ffsplit_launch_count.argtypes = [vp]
    lib.ffsplit_launch_count.restype = i64
    lib.ffsplit_last_error.argtypes = [vp]
    lib.ffsplit_last_error.restype = C.c_char_p
    lib.ffsplit_version.argtypes = []
    lib.ffsplit_version.restype = i32
    for name in EXPORTS:
        fn = getattr(lib, name)
        if name not in ("ffsplit_launch_count", "ffsplit_last_error", "ffsplit_version"):
            fn.restype = C.c_int
    if path is None:
        _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _status_words(workspace: torch.Tensor) -> torch.Tensor:
    """Where a workspace holds the first condition that a kernel recorded: its code, a detail, the kernel's number."""
    return workspace.reshape(-1).view(torch.uint8)[:12].view(torch.int32)


class GradList:
    """The tensors whose gradients are clipped together, as the array ffsplit_grad_norm() / ffsplit_grad_clip() take.
    `out` holds where the clipped gradients go, tensor by tensor; without it they replace the gradients.  The list
    keeps the tensors alive and names their memory: make a new one when a gradient moves to another buffer."""

    def __init__(self, device: int, grads, out=None):
        self.grads, self.out = list(grads), list(grads) if out is None else list(out)
        if len(self.grads) != len(self.out):
            raise FFSplitError(2, "grad_list", "as many outputs as gradients are needed")
        words = []
        for g, o in zip(self.grads, self.out):
            kind, n = DTYPE_IDS.get(g.dtype), g.numel()
            if kind is None or o.dtype is not g.dtype:
                raise FFSplitError(4, "grad_list", "gradients are float32 or bfloat16, and outputs of the same type")
            if o.numel() != n or not g.is_contiguous() or not o.is_contiguous():
                raise FFSplitError(2, "grad_list", "tensors must be contiguous, and outputs as long as the gradients")
            if g.get_device() != device or o.get_device() != device:
                raise FFSplitError(1, "grad_list", f"tensors must be on cuda:{device}")
            words += (g.data_ptr(), o.data_ptr(), n, kind)
        # ffsplit_grad_tensor is four 8-byte words (the type, and padding, in the last)
        self.count = len(self.grads)
        self.array = (C.c_int64 * max(4, len(words)))(*words)


class MuonList:
    """The matrices that one call updates (or orthogonalises), as the array ffsplit_muon_step() takes.  `step` and `decay`
    are numbers, or one for each matrix.  Without out_weights and out_momenta both are updated in place.  The list keeps
    the tensors alive and names their memory: make a new one when a tensor moves or a rate changes."""

    def __init__(self, device: int, grads, weights=None, momenta=None, step=0.0, decay=0.0, out=None, out_momenta=None):
        self.grads, n = list(grads), len(grads)
        whole = lambda v: [None] * n if v is None else list(v)  # noqa: E731
        self.weights, self.momenta = whole(weights), whole(momenta)
        self.out = list(self.weights if out is None else out)
        self.out_momenta = list(self.momenta if out_momenta is None else out_momenta)
        rates = [list(v) if isinstance(v, (list, tuple)) else [v] * n for v in (step, decay)]
        if any(len(v) != n for v in (self.weights, self.momenta, self.out, self.out_momenta, *rates)):
            raise FFSplitError(2, "muon_list", "lists must be of the same length")
        written = [v.data_ptr() for v in self.out + self.out_momenta if v is not None]
        if len(set(written)) < len(written):
            raise FFSplitError(1, "muon_list", "two matrices of one call write to the same memory")
        self.count = n
        self.array = (MuonTensor * max(1, n))()
        for e, g, w, m, o, mo, s, d in zip(self.array, self.grads, self.weights, self.momenta, self.out, self.out_momenta, *rates):
            if g.dtype not in DTYPE_IDS or o is None or o.dtype not in DTYPE_IDS or (w is not None and w.dtype is not o.dtype):
                raise FFSplitError(4, "muon_list", "gradients and weights are float32 or bfloat16, outputs of the weights' type")
            if any(v is not None and v.dtype is not torch.float32 for v in (m, mo)):
                raise FFSplitError(4, "muon_list", "momentum is float32")
            if (m is None) != (mo is None):
                raise FFSplitError(1, "muon_list", "momentum goes with an output for it")
            if g.dim() != 2:
                raise FFSplitError(2, "muon_list", "matrices have two dimensions")
            for v in (g, w, m, o, mo):
                if v is not None and (v.shape != g.shape or not v.is_contiguous()):
                    raise FFSplitError(2, "muon_list", "a matrix's tensors must be contiguous and of one shape")
            if any(v is not None and v.get_device() != device for v in (g, w, m, o, mo)):
                raise FFSplitError(1, "muon_list", f"tensors must be on cuda:{device}")
            e.grad, e.out, e.rows, e.cols = g.data_ptr(), o.data_ptr(), g.shape[0], g.shape[1]
            e.weight = None if w is None else w.data_ptr()
            e.momentum, e.momentum_out = (None, None) if m is None else (m.data_ptr(), mo.data_ptr())
            e.grad_dtype, e.weight_dtype, e.step, e.decay = DTYPE_IDS[g.dtype], DTYPE_IDS[o.dtype], s, d


def make_shape(d: int, m: int, act, dtype) -> Shape:
    a = ACT_IDS[act] if isinstance(act, str) else int(act)
    t = DTYPE_IDS[dtype] if isinstance(dtype, torch.dtype) else int(dtype)
    return Shape(d, m, a, t)


class Context:
    """One ffsplit_ctx bound to a CUDA device, plus the torch tensors that back
    its workspace.  Methods mirror the C entry points one to one."""

    _in_graph = False      # a captured graph uses the workspace
    _retired = ()          # workspaces before it that captured graphs use

    def __init__(self, device: int = 0):
        self.lib = load_library()
        self.device = device
        torch.cuda.set_device(device)
        h = C.c_void_p()
        rc = self.lib.ffsplit_create(C.byref(h), device)
        if rc != OK:
            raise FFSplitError(rc, "ffsplit_create")
        self.h = h
        self._ws = None

    def close(self):
        if getattr(self, "h", None):
            self.lib.ffsplit_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self, stream) -> int:
        """The handle of `stream`, or of the device's current stream (without making a Stream object of it: that takes the
        interpreter longer than a launch).  Every call that launches asks here, and one that is captured ties the workspace
        to its graph."""
        if torch._C._cuda_isCurrentStreamCapturing():
            self._in_graph = True
        return torch._C._cuda_getCurrentRawStream(self.device) if stream is None else stream.cuda_stream

    def _check(self, rc: int, where: str):
        if rc != OK:
            raise FFSplitError(rc, where, (self.lib.ffsplit_last_error(self.h) or b"").decode())

    # ------------------------------------------------------------------ workspace
    def workspace_size(self, shape: Shape, T_fwd: int, T_cal: int, k: int, r: int) -> int:
        n = C.c_size_t()
        self._check(self.lib.ffsplit_workspace_size(C.byref(shape), T_fwd, T_cal, k, r, C.byref(n)),
                    "ffsplit_workspace_size")
        return n.value

    def set_workspace(self, tensor: torch.Tensor):
        """ffsplit_set_workspace, once the device is idle: torch hands out memory that work queued on some stream may still
        use, and takes back the workspace before this one, which calls still running may use.  Not while a graph is captured.
        A workspace that a captured graph uses stays allocated as long as the context lives."""
        if torch.cuda.is_current_stream_capturing():
            raise FFSplitError(1, "ffsplit_set_workspace", "a workspace cannot be set while a graph is captured: set one of "
                                                           "sufficient size before")
        torch.cuda.synchronize(self.device)
        self._check(self.lib.ffsplit_set_workspace(self.h, _ptr(tensor), tensor.numel() * tensor.element_size()),
                    "ffsplit_set_workspace")
        if self._in_graph and self._ws is not tensor:
            self._retired, self._in_graph = (*self._retired, self._ws), False
        self._ws = tensor

    def ensure_workspace(self, nbytes: int):
        """Allocate (with torch) and install a workspace of at least nbytes.  A device-side condition that poll() has not
        reported yet moves on to it."""
        old = self._ws
        if old is not None and old.numel() >= nbytes:
            return
        new = torch.empty(nbytes, dtype=torch.uint8, device=f"cuda:{self.device}")
        self.set_workspace(new)
        if old is not None:
            _status_words(new).copy_(_status_words(old))
            _status_words(old).zero_()
            torch.cuda.synchronize(self.device)      # (the next call may be on another stream)

    # ------------------------------------------------------------------ entry points
    def score(self, shape: Shape, W1, b1, W2, X, energy, scores=None, mode=SCORE_EQ3, accumulate=False, W1u=None,
              stream=None):
        w = Weights(_ptr(W1), _ptr(W1u), _ptr(b1), _ptr(W2), None)
        self._check(self.lib.ffsplit_score(self.h, C.byref(shape), C.byref(w), _ptr(X), X.shape[0], int(mode),
                                           int(bool(accumulate)), _ptr(energy), _ptr(scores), self._stream(stream)),
                    "ffsplit_score")

    def score_activations(self, shape: Shape, H, W2, energy, scores=None, mode=SCORE_EQ3, accumulate=False,
                          stream=None):
        """ffsplit_score_activations: Eq. 3 from a stored activation matrix H [T, m]."""
        self._check(self.lib.ffsplit_score_activations(self.h, C.byref(shape), _ptr(H), H.shape[0], _ptr(W2), mode,
                                                       1 if accumulate else 0, _ptr(energy), _ptr(scores),
                                                       self._stream(stream)), "ffsplit_score_activations")

    def select(self, scores, k: int, heavy_idx, light_idx=None, stream=None):
        self._check(self.lib.ffsplit_select(self.h, _ptr(scores), scores.numel(), k, _ptr(heavy_idx), _ptr(light_idx),
                                            self._stream(stream)), "ffsplit_select")

    def pack_size(self, shape: Shape, k: int, r: int):
        a, b = C.c_size_t(), C.c_size_t()
        self._check(self.lib.ffsplit_pack_size(C.byref(shape), k, r, C.byref(a), C.byref(b)), "ffsplit_pack_size")
        return a.value, b.value

    def pack(self, shape: Shape, W1, b1, W2, b2, heavy_idx, k: int, factors: Optional[dict], blob, W1u=None,
             stream=None):
        w = Weights(_ptr(W1), _ptr(W1u), _ptr(b1), _ptr(W2), _ptr(b2))
        fp = None
        if factors is not None:
            f = Factors(_ptr(factors["A1"]), _ptr(factors["B1"]), _ptr(factors.get("A1u")), _ptr(factors.get("B1u")),
                        _ptr(factors["A2"]), _ptr(factors["B2"]), int(factors["A1"].shape[1]))
            fp = C.byref(f)
        self._check(self.lib.ffsplit_pack(self.h, C.byref(shape), C.byref(w), _ptr(heavy_idx), k, fp, _ptr(blob),
                                          blob.numel() * blob.element_size(), self._stream(stream)), "ffsplit_pack")

    def blob_open(self, blob, stream=None):
        self._check(self.lib.ffsplit_blob_open(self.h, _ptr(blob), blob.numel() * blob.element_size(),
                                               self._stream(stream)), "ffsplit_blob_open")

    def blob_close(self, blob):
        self._check(self.lib.ffsplit_blob_close(self.h, _ptr(blob)), "ffsplit_blob_close")

    def score_host(self, shape: Shape, W1, b1, W2, X_host, energy, scores=None, mode=SCORE_EQ3, accumulate=False,
                   W1u=None, stream=None):
        """ffsplit_score_host: calibration tokens in (pinned) host memory, staged through the workspace in chunks."""
        w = Weights(_ptr(W1), _ptr(W1u), _ptr(b1), _ptr(W2), None)
        self._check(self.lib.ffsplit_score_host(self.h, C.byref(shape), C.byref(w), _ptr(X_host), X_host.shape[0],
                                                int(mode), int(bool(accumulate)), _ptr(energy), _ptr(scores),
                                                self._stream(stream)), "ffsplit_score_host")

    def score_finalize(self, shape: Shape, W2, energy, scores, mode=SCORE_EQ3, stream=None):
        """ffsplit_score_finalize: scores from a complete energy vector (after a sharded or multi-call accumulation)."""
        self._check(self.lib.ffsplit_score_finalize(self.h, C.byref(shape), _ptr(W2), int(mode), _ptr(energy),
                                                    _ptr(scores), self._stream(stream)), "ffsplit_score_finalize")

    @staticmethod
    def _blob_array(blobs):
        arr = (C.c_void_p * len(blobs))(*[b.data_ptr() for b in blobs])
        return arr

    def stack_workspace_size(self, blobs, T: int) -> int:
        n = C.c_size_t()
        self._check(self.lib.ffsplit_stack_workspace_size(self.h, self._blob_array(blobs), len(blobs), T, C.byref(n)),
                    "ffsplit_stack_workspace_size")
        return n.value

    def forward_stack(self, blobs, X, Y, stream=None):
        self._check(self.lib.ffsplit_forward_stack(self.h, self._blob_array(blobs), len(blobs), _ptr(X), X.shape[0],
                                                   _ptr(Y), self._stream(stream)), "ffsplit_forward_stack")

    def forward_stack_host(self, blobs, X_host, Y_host, stream=None):
        self._check(self.lib.ffsplit_forward_stack_host(self.h, self._blob_array(blobs), len(blobs), _ptr(X_host),
                                                        X_host.shape[0], _ptr(Y_host), self._stream(stream)),
                    "ffsplit_forward_stack_host")

    # ------------------------------------------------------------------ the transformer block around the FFN
    def encoder_desc(self, batch: int, seq: int, heads: int, Wqkv_t, bqkv, Wo_t, bo, ln1, ln2, eps: float, ffn_blob):
        """ffsplit_encoder_layer from device tensors; ln1, ln2 = (gamma, beta).  The tensors must stay alive."""
        return EncoderLayer(batch, seq, heads, Wqkv_t.data_ptr(), bqkv.data_ptr(), Wo_t.data_ptr(), bo.data_ptr(),
                            ln1[0].data_ptr(), ln1[1].data_ptr(), ln2[0].data_ptr(), ln2[1].data_ptr(), eps,
                            ffn_blob.data_ptr())

    def encoder_workspace_size(self, layer: "EncoderLayer") -> int:
        n = C.c_size_t()
        self._check(self.lib.ffsplit_encoder_workspace_size(self.h, C.byref(layer), C.byref(n)), "ffsplit_encoder_workspace_size")
        return n.value

    def encoder_forward(self, layer: "EncoderLayer", X, Y, stream=None):
        self._check(self.lib.ffsplit_encoder_forward(self.h, C.byref(layer), _ptr(X), _ptr(Y), self._stream(stream)),
                    "ffsplit_encoder_forward")

    # ------------------------------------------------------------------ on-device light factors (Section 5.1.1)
    def factor_workspace_size(self, shape: Shape, k: int, r: int) -> int:
        n = C.c_size_t()
        self._check(self.lib.ffsplit_factor_workspace_size(C.byref(shape), k, r, C.byref(n)), "ffsplit_factor_workspace_size")
        return n.value

    def factor_light(self, shape: Shape, W1, W2, light_idx, k: int, r: int, iters: int, start, W1u=None, stream=None) -> dict:
        """ffsplit_factor_light: rank-r factors of the light slices as a dict ready for pack().  `start` is the
        [n, r, d] starting basis (n = 2, or 3 with W1u) in the layer's dtype."""
        d, m = shape.d, shape.m
        ml = m - k
        dev, dt = W1.device, W1.dtype
        f = {"A1": torch.empty(d, r, dtype=dt, device=dev), "B1": torch.empty(r, ml, dtype=dt, device=dev),
             "A2": torch.empty(ml, r, dtype=dt, device=dev), "B2": torch.empty(r, d, dtype=dt, device=dev)}
        if W1u is not None:
            f["A1u"] = torch.empty(d, r, dtype=dt, device=dev)
            f["B1u"] = torch.empty(r, ml, dtype=dt, device=dev)
        w = Weights(_ptr(W1), _ptr(W1u), None, _ptr(W2), None)
        self._check(self.lib.ffsplit_factor_light(self.h, C.byref(shape), C.byref(w), _ptr(light_idx), k, r, iters,
                                                  _ptr(start), _ptr(f["A1"]), _ptr(f["B1"]), _ptr(f["A2"]), _ptr(f["B2"]),
                                                  _ptr(f.get("A1u")), _ptr(f.get("B1u")), self._stream(stream)),
                    "ffsplit_factor_light")
        return f

    # ------------------------------------------------------------------ quantised split (Section 5.2)
    def quant_pack_size(self, shape: Shape, k: int):
        a, b = C.c_size_t(), C.c_size_t()
        self._check(self.lib.ffsplit_quant_pack_size(C.byref(shape), k, C.byref(a), C.byref(b)), "ffsplit_quant_pack_size")
        return a.value, b.value

    def quant_workspace_size(self, shape: Shape, k: int) -> int:
        n = C.c_size_t()
        self._check(self.lib.ffsplit_quant_workspace_size(C.byref(shape), k, C.byref(n)), "ffsplit_quant_workspace_size")
        return n.value

    def quant_pack(self, shape: Shape, W1, b1, W2, b2, heavy_idx, k: int, light_idx, blob, W1u=None, stream=None):
        w = Weights(_ptr(W1), _ptr(W1u), _ptr(b1), _ptr(W2), _ptr(b2))
        self._check(self.lib.ffsplit_quant_pack(self.h, C.byref(shape), C.byref(w), _ptr(heavy_idx), k, _ptr(light_idx),
                                                _ptr(blob), blob.numel() * blob.element_size(), self._stream(stream)),
                    "ffsplit_quant_pack")

    def quant_blob_open(self, blob, stream=None):
        self._check(self.lib.ffsplit_quant_blob_open(self.h, _ptr(blob), blob.numel() * blob.element_size(),
                                                     self._stream(stream)), "ffsplit_quant_blob_open")

    def quant_unpack(self, blob, which: int, rows: int, cols: int, stream=None):
        """-> (codes uint8 [rows, cols], scale float32 [rows, ceil(cols / 128)], lo likewise) of one packed matrix."""
        dev = blob.device
        codes = torch.zeros(rows, cols, dtype=torch.uint8, device=dev)
        ng = (cols + 127) // 128
        scale = torch.zeros(rows, ng, dtype=torch.float32, device=dev)
        lo = torch.zeros(rows, ng, dtype=torch.float32, device=dev)
        self._check(self.lib.ffsplit_quant_unpack(self.h, _ptr(blob), which, _ptr(codes), _ptr(scale), _ptr(lo),
                                                  self._stream(stream)), "ffsplit_quant_unpack")
        return codes, scale, lo

    def quant_forward(self, blob, X, Y, stream=None):
        self._check(self.lib.ffsplit_quant_forward(self.h, _ptr(blob), _ptr(X), X.shape[0], _ptr(Y), self._stream(stream)),
                    "ffsplit_quant_forward")

    # ------------------------------------------------------------------ training
    # (These calls are made per layer and step, and a small layer takes the GPU no longer than the interpreter takes to
    # get here: the checks below are written to cost little.)
    def _operand(self, where: str, name: str, t, dtype, dims, optional: bool = True):
        """Address of one tensor of a training call, checked against what the layer says it has to be."""
        if t is None:
            if optional:
                return None
            raise FFSplitError(1, where, f"{name} is missing")
        if t.dtype is not dtype:
            raise FFSplitError(4, where, f"{name} is {t.dtype}, which is not the layer's type")
        if t.shape != dims or not t.is_contiguous():
            raise FFSplitError(2, where, f"{name} must be contiguous and of shape {dims}")
        if t.get_device() != self.device:
            raise FFSplitError(1, where, f"{name} must be on cuda:{self.device}")
        return t.data_ptr()

    def _saved(self, where: str, saved):
        """Address and size of what the forward pass keeps."""
        if saved is None:
            return None, 0
        if saved.get_device() != self.device or not saved.is_contiguous():
            raise FFSplitError(1, where, f"saved must be contiguous and on cuda:{self.device}")
        return saved.data_ptr(), saved.nbytes

    def _train_weights(self, where, shape, W1, W1u, b1, W2, b2):
        d, m, op, dt = shape.d, shape.m, self._operand, DTYPES[shape.dtype]
        return Weights(op(where, "W1", W1, dt, (d, m), False), op(where, "W1u", W1u, dt, (d, m)), op(where, "b1", b1, dt, (m,)),
                       op(where, "W2", W2, dt, (m, d), False), op(where, "b2", b2, dt, (d,)))

    def train_sizes(self, shape: Shape, T: int):
        """-> (bytes of `saved`, bytes of workspace) that train_forward / train_backward need for T tokens."""
        a, b = C.c_size_t(), C.c_size_t()
        rc = self.lib.ffsplit_train_sizes(C.byref(shape), T, C.byref(a), C.byref(b))
        if rc != OK:
            raise FFSplitError(rc, "ffsplit_train_sizes")
        return a.value, b.value

    def train_forward(self, shape: Shape, W1, b1, W2, b2, X, Y, saved=None, W1u=None, stream=None):
        """ffsplit_train_forward: Y from the row-major weights; `saved` (a byte tensor) is written for train_backward()."""
        where, T, d, dt = "ffsplit_train_forward", X.shape[0], shape.d, DTYPES[shape.dtype]
        w = self._train_weights(where, shape, W1, W1u, b1, W2, b2)
        rc = self.lib.ffsplit_train_forward(
            self.h, shape, w, self._operand(where, "X", X, dt, (T, d), False), T, *self._saved(where, saved),
            self._operand(where, "Y", Y, dt, (T, d), False), self._stream(stream))
        if rc:
            self._check(rc, where)

    def train_backward(self, shape: Shape, W1, b1, W2, X, saved, dY, dX=None, dW1=None, db1=None, dW2=None, db2=None,
                       W1u=None, dW1u=None, stream=None):
        """ffsplit_train_backward: writes the gradients that are given (None: not wanted)."""
        where, T, d, m, op, dt = "ffsplit_train_backward", X.shape[0], shape.d, shape.m, self._operand, DTYPES[shape.dtype]
        w = self._train_weights(where, shape, W1, W1u, None, W2, None)
        g = TrainGrads(op(where, "dX", dX, dt, (T, d)), op(where, "dW1", dW1, dt, (d, m)), op(where, "dW1u", dW1u, dt, (d, m)),
                       op(where, "db1", db1, dt, (m,)), op(where, "dW2", dW2, dt, (m, d)), op(where, "db2", db2, dt, (d,)))
        rc = self.lib.ffsplit_train_backward(
            self.h, shape, w, op(where, "X", X, dt, (T, d), False), T, *self._saved(where, saved),
            op(where, "dY", dY, dt, (T, d), False), g, self._stream(stream))
        if rc:
            self._check(rc, where)

    def grad_list(self, grads, out=None) -> "GradList":
        return GradList(self.device, grads, out)

    def grad_workspace_size(self, count: int) -> int:
        n = C.c_size_t()
        self._check(self.lib.ffsplit_grad_workspace_size(count, C.byref(n)), "ffsplit_grad_workspace_size")
        return n.value

    def _norm_ptr(self, where, norm):
        if norm.dtype != torch.float32 or norm.numel() != 1 or norm.device.type != "cuda" or norm.device.index != self.device:
            raise FFSplitError(2, where, f"norm must be one float32 on cuda:{self.device}")
        return _ptr(norm)

    def grad_norm(self, grads: "GradList", norm, stream=None):
        """ffsplit_grad_norm: norm[0] = the 2-norm of all gradients of the list."""
        self._check(self.lib.ffsplit_grad_norm(self.h, C.byref(grads.array), grads.count, self._norm_ptr("ffsplit_grad_norm", norm),
                                               self._stream(stream)), "ffsplit_grad_norm")

    def clip_grads(self, grads: "GradList", max_norm: float, norm, stream=None):
        """ffsplit_grad_clip: the norm, then every gradient times min(1, max_norm / (norm + 1e-6))."""
        self._check(self.lib.ffsplit_grad_clip(self.h, C.byref(grads.array), grads.count, max_norm,
                                               self._norm_ptr("ffsplit_grad_clip", norm), self._stream(stream)), "ffsplit_grad_clip")

    # ------------------------------------------------------------------ orthogonalised momentum
    def muon_list(self, weights, grads, momenta, step, decay=0.0, out_weights=None, out_momenta=None) -> "MuonList":
        return MuonList(self.device, grads, weights, momenta, step, decay, out_weights, out_momenta)

    def orthogonal_list(self, matrices, out) -> "MuonList":
        return MuonList(self.device, matrices, out=out)

    def muon_workspace_size(self, tensors: "MuonList") -> int:
        n = C.c_size_t()
        self._check(self.lib.ffsplit_muon_workspace_size(C.byref(tensors.array), tensors.count, C.byref(n)), "ffsplit_muon_workspace_size")
        return n.value

    def muon_step(self, tensors: "MuonList", beta: float = 0.95, nesterov: bool = True, coefficients=None, iterations: int = 5,
                  stream=None):
        """ffsplit_muon_step: momentum, its orthogonal factor, decay and step for every matrix of the list.  `coefficients`:
        one (a, b, c) to an iteration, in place of `iterations` times (3.4445, -4.7750, 2.0315)."""
        c = None
        if coefficients is not None:
            iterations = len(coefficients)
            if any(len(v) != 3 for v in coefficients):
                raise FFSplitError(2, "ffsplit_muon_step", "three coefficients to an iteration")
            c = (C.c_float * max(3, 3 * iterations))(*[x for v in coefficients for x in v])
        self._check(self.lib.ffsplit_muon_step(self.h, C.byref(tensors.array), tensors.count, beta, int(bool(nesterov)),
                                               c, iterations, self._stream(stream)), "ffsplit_muon_step")

    def orthogonalize(self, tensors: "MuonList", coefficients=None, iterations: int = 5, stream=None):
        """ffsplit_muon_step on a list without weights and momentum: out = the orthogonal factor of every matrix."""
        self.muon_step(tensors, 0.0, False, coefficients, iterations, stream)

    # ------------------------------------------------------------------ low-rank adapters beside a shared projection
    def adapter_workspace_size(self, projection: Projection, n: int, r: int, T: int) -> int:
        b = C.c_size_t()
        rc = self.lib.ffsplit_adapter_workspace_size(C.byref(projection), n, r, T, C.byref(b))
        if rc != OK:
            raise FFSplitError(rc, "ffsplit_adapter_workspace_size")
        return b.value

    def _adapters(self, where, p, A, B, index, scale, T):
        if A.dim() != 3:
            raise FFSplitError(2, where, "A must be of shape (adapters, inner, rank)")
        n, r, dt, op = A.shape[0], A.shape[2], DTYPES[p.dtype], self._operand
        return Adapters(op(where, "A", A, dt, (n, p.inner, r), False), op(where, "B", B, dt, (n, r, p.outer), False),
                        op(where, "scale", scale, torch.float32, (n,)), op(where, "index", index, torch.int32, (T,), False), n, r)

    def adapter_forward(self, projection: Projection, X, A, B, index, Y, W=None, b=None, base=None, scale=None, stream=None):
        """ffsplit_adapter_forward: Y = (X W + b, or base, or nothing) + scale_i (X A_i) B_i, i = index[t] (negative: none)."""
        where, T, p, op = "ffsplit_adapter_forward", X.shape[0], projection, self._operand
        dt, k, m = DTYPES[p.dtype], p.inner, p.outer
        rc = self.lib.ffsplit_adapter_forward(
            self.h, p, op(where, "W", W, dt, (k, m)), op(where, "b", b, dt, (m,)), op(where, "base", base, dt, (T, m)),
            self._adapters(where, p, A, B, index, scale, T), op(where, "X", X, dt, (T, k), False), T,
            op(where, "Y", Y, dt, (T, m), False), self._stream(stream))
        if rc:
            self._check(rc, where)

    def adapter_backward(self, projection: Projection, X, A, B, index, dY, W=None, base=None, scale=None, dX=None, dA=None,
                         dB=None, stream=None):
        """ffsplit_adapter_backward: writes the gradients that are given (None: not wanted)."""
        where, T, p, op = "ffsplit_adapter_backward", X.shape[0], projection, self._operand
        dt, k, m = DTYPES[p.dtype], p.inner, p.outer
        a = self._adapters(where, p, A, B, index, scale, T)
        rc = self.lib.ffsplit_adapter_backward(
            self.h, p, op(where, "W", W, dt, (k, m)), op(where, "base", base, dt, (T, k)), a, op(where, "X", X, dt, (T, k), False),
            T, op(where, "dY", dY, dt, (T, m), False),
            AdapterGrads(op(where, "dX", dX, dt, (T, k)), op(where, "dA", dA, dt, (a.n, k, a.r)), op(where, "dB", dB, dt, (a.n, a.r, m))),
            self._stream(stream))
        if rc:
            self._check(rc, where)

    def debug_wait_timeout(self, limit_cycles: int, stream=None):
        self._check(self.lib.ffsplit_debug_wait_timeout(self.h, int(limit_cycles), self._stream(stream)),
                    "ffsplit_debug_wait_timeout")

    def blob_section(self, blob, which: int):
        off, r, c, ld = C.c_size_t(), C.c_int64(), C.c_int64(), C.c_int64()
        self._check(self.lib.ffsplit_blob_section(self.h, _ptr(blob), which, C.byref(off), C.byref(r), C.byref(c),
                                                  C.byref(ld)), "ffsplit_blob_section")
        return off.value, r.value, c.value, ld.value

    def forward(self, blob, X, Y, stream=None):
        self._check(self.lib.ffsplit_forward(self.h, _ptr(blob), _ptr(X), X.shape[0], _ptr(Y), self._stream(stream)),
                    "ffsplit_forward")

    def forward_dense(self, shape: Shape, W1, b1, W2, b2, X, Y, W1u=None, stream=None):
        """ffsplit_forward_dense: the unsplit FFN from the row-major weights (packed into the workspace per call)."""
        w = Weights(_ptr(W1), _ptr(W1u), _ptr(b1), _ptr(W2), _ptr(b2))
        self._check(self.lib.ffsplit_forward_dense(self.h, C.byref(shape), C.byref(w), _ptr(X), X.shape[0], _ptr(Y),
                                                   self._stream(stream)), "ffsplit_forward_dense")

    def forward_noalloc(self, blob, X, Y, stream=None):
        """ffsplit_forward_noalloc: up to 8 tokens, bf16, scratch built into the library (no workspace needed)."""
        self._check(self.lib.ffsplit_forward_noalloc(self.h, _ptr(blob), _ptr(X), X.shape[0], _ptr(Y),
                                                     self._stream(stream)), "ffsplit_forward_noalloc")

    def forward_host(self, blob, X_host, Y_host, stream=None):
        self._check(self.lib.ffsplit_forward_host(self.h, _ptr(blob), _ptr(X_host), X_host.shape[0], _ptr(Y_host),
                                                  self._stream(stream)), "ffsplit_forward_host")

    def poll(self, stream=None):
        """ffsplit_poll, and the same for workspaces that only captured graphs still use."""
        self._check(self.lib.ffsplit_poll(self.h, self._stream(stream)), "ffsplit_poll")
        for ws in self._retired:
            code, detail, kernel = _status_words(ws).tolist()
            if code:
                ws.reshape(-1).view(torch.uint8)[:65536].zero_()
                torch.cuda.synchronize(self.device)
                raise FFSplitError(code, "ffsplit_poll", f"device status {code} (detail {detail}, kernel {kernel}, a captured graph's workspace)")

    def profile_begin(self):
        self._check(self.lib.ffsplit_profile_begin(self.h), "ffsplit_profile_begin")

    def profile_end(self, kernel_class: int = 0, stream=None):
        """-> (launches, total milliseconds, total algorithmic work) of one kernel class."""
        n, ms, work = C.c_int32(), C.c_double(), C.c_double()
        self._check(self.lib.ffsplit_profile_end(self.h, self._stream(stream), kernel_class, C.byref(n), C.byref(ms),
                                                 C.byref(work)), "ffsplit_profile_end")
        return n.value, ms.value, work.value

    def launch_count(self) -> int:
        return int(self.lib.ffsplit_launch_count(self.h))


def read_section(ctx: Context, blob: torch.Tensor, which: int, dtype: torch.dtype) -> torch.Tensor:
    """View of one matrix inside a packed blob (for inspection and tests)."""
    off, rows, cols, ld = ctx.blob_section(blob, which)
    es = torch.empty((), dtype=dtype).element_size()
    raw = blob.view(torch.uint8)[off: off + rows * ld * es]
    return raw.view(dtype).view(rows, ld)[:, :cols]
