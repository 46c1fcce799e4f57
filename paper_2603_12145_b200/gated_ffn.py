"""ctypes binding of libgated_ffn_b200.so: the entry points of include/gated_ffn.h, and a
small wrapper that owns the handle, checks tensors and allocates outputs with torch.
No CPU path."""
from __future__ import annotations

import ctypes
import os

from . import build as _build

EXPORTS = ("gated_ffn_create", "gated_ffn_destroy", "gated_ffn_set_stream", "gated_ffn_workspace_bytes",
           "gated_ffn_pre_bytes", "gated_ffn_forward", "gated_ffn_backward", "gated_ffn_status", "gated_ffn_launch_count",
           "gated_ffn_strerror")

ACTIVATIONS = {"silu": 0, "gelu": 1}


class GatedFfnError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (code %d)" % (where, strerror(code), code))


_lib = None


def load(build_if_missing: bool = False):
    """Load libgated_ffn_b200.so.  Raises if it is missing (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.GATED_FFN_LIB
    if build_if_missing:
        _build.build_one("libgated_ffn_b200.so")
    if not os.path.exists(path):
        raise ImportError("CUDA library %s is not built; run `python -m paper_2603_12145_b200.build`"
                          " (needs nvcc). There is no CPU fallback." % path)
    L = ctypes.CDLL(path)
    vp, i32, i64, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    L.gated_ffn_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32, i32]
    L.gated_ffn_destroy.argtypes = [vp]
    L.gated_ffn_set_stream.argtypes = [vp, vp]
    L.gated_ffn_workspace_bytes.argtypes = [vp, i64, i32]
    L.gated_ffn_pre_bytes.argtypes = [vp, i64]
    L.gated_ffn_forward.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, i64, vp, size, i64]
    L.gated_ffn_backward.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, vp, size, i64]
    L.gated_ffn_status.argtypes = [vp]
    L.gated_ffn_launch_count.argtypes = [vp]
    L.gated_ffn_strerror.argtypes = [i32]
    for name in EXPORTS:
        getattr(L, name).restype = i32
    L.gated_ffn_workspace_bytes.restype = size
    L.gated_ffn_pre_bytes.restype = size
    L.gated_ffn_launch_count.restype = i64
    L.gated_ffn_strerror.restype = ctypes.c_char_p
    _lib = L
    return L


def strerror(code: int) -> str:
    return load().gated_ffn_strerror(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise GatedFfnError(code, where)


def gated_ffn_create(model: int, hidden: int, activation: int, type_: int) -> int:
    h = ctypes.c_void_p()
    _check(load().gated_ffn_create(ctypes.byref(h), model, hidden, activation, type_), "gated_ffn_create")
    return h.value


def gated_ffn_destroy(h: int) -> None:
    _check(load().gated_ffn_destroy(h), "gated_ffn_destroy")


def gated_ffn_status(h: int) -> None:
    _check(load().gated_ffn_status(h), "gated_ffn_status")


def gated_ffn_launch_count(h: int) -> int:
    return int(load().gated_ffn_launch_count(h))


# ---- a small owner of the handle ----------------------------------------------------

class GatedFfn:
    """The block for one layer's sizes.  Tensors are torch CUDA tensors of the handle's dtype:
    x, dy [n, model] with a contiguous last dimension and a row stride that is a multiple of 8;
    w_in [2 * hidden, model] (gate rows first) and w_out [model, hidden] contiguous.  Calls
    enqueue on the current stream of the device, whichever device is current.  One thread at a
    time.  A tensor that does not fit raises ValueError, a refusal by the library GatedFfnError."""

    def __init__(self, model: int, hidden: int, activation: str = "silu", dtype=None, device: str = "cuda:0"):
        import torch
        self.torch = torch
        self.dtype = torch.bfloat16 if dtype is None else dtype
        types = {torch.bfloat16: 0, torch.float16: 1}
        if self.dtype not in types:
            raise ValueError("dtype must be bfloat16 or float16")
        if activation not in ACTIVATIONS:
            raise ValueError("activation must be one of %s" % (tuple(ACTIVATIONS),))
        self.model, self.hidden, self.activation = int(model), int(hidden), activation
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("device must be a CUDA device")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        # the current stream's handle without building a Stream object: a single token is short
        self._current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
        self._lib = load()
        self._on = None                   # the stream that the handle was last given
        with torch.cuda.device(self.device):
            self.h = gated_ffn_create(self.model, self.hidden, ACTIVATIONS[activation], types[self.dtype])

    def close(self):
        if getattr(self, "h", None):
            with self.torch.cuda.device(self.device):
                gated_ffn_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launches(self) -> int:
        return gated_ffn_launch_count(self.h)

    def _stream(self):
        stream = self._current(self._index)
        if stream != self._on:
            self._lib.gated_ffn_set_stream(self.h, stream)
            self._on = stream

    def _bad(self, name, v, want):
        raise ValueError("%s must be %s on %s, got %s %s on %s with strides %s"
                         % (name, want, self.device, v.dtype, tuple(v.shape), v.device, v.stride()))

    def _rows(self, name, v, n):
        if (v.dtype is not self.dtype or v.shape != (n, self.model) or v.get_device() != self._index or v.stride(1) != 1):
            self._bad(name, v, "%s [%d, %d] with a contiguous last dimension" % (self.dtype, n, self.model))
        return v.data_ptr()

    def _dense(self, name, v, shape):
        if v.dtype is not self.dtype or v.shape != shape or v.get_device() != self._index or not v.is_contiguous():
            self._bad(name, v, "contiguous %s %s" % (self.dtype, shape))
        return v.data_ptr()

    def _stride(self, v):
        return v.stride(0) if v.shape[0] > 1 else self.model     # of a single row any stride is as good

    def _empty(self, *shape):
        return self.torch.empty(shape, dtype=self.dtype, device=self.device)

    def _scratch(self, n, backward):
        size = self._lib.gated_ffn_workspace_bytes(self.h, n, backward)
        return (self.torch.empty((size,), dtype=self.torch.uint8, device=self.device) if size else None), size

    def saved(self, n: int):
        """Buffers in which forward() leaves what backward() needs: (pre-activations, hidden)."""
        t = self.torch
        return (t.empty((self._lib.gated_ffn_pre_bytes(self.h, n),), dtype=t.uint8, device=self.device),
                self._empty(n, self.hidden))

    def _saved(self, saved, n):
        pre, hidden = saved
        need = self._lib.gated_ffn_pre_bytes(self.h, n)
        if pre.dtype is not self.torch.uint8 or pre.shape != (need,) or pre.device != self.device:
            self._bad("saved[0]", pre, "uint8 (%d,)" % need)
        return pre.data_ptr(), self._dense("saved[1]", hidden, (n, self.hidden))

    def forward(self, x, w_in, w_out, saved=None, out=None):
        n = x.shape[0]
        if out is None:
            out = self._empty(n, self.model)
        if saved is None:
            kept = self._empty(n, self.hidden)
            pre, hidden = None, kept.data_ptr()
        else:
            pre, hidden = self._saved(saved, n)
        scratch, size = self._scratch(n, 0)
        self._stream()
        _check(self._lib.gated_ffn_forward(
            self.h, self._rows("x", x, n), self._stride(x), self._dense("w_in", w_in, (2 * self.hidden, self.model)),
            self._dense("w_out", w_out, (self.model, self.hidden)), pre, hidden, self._rows("out", out, n), self._stride(out),
            None if scratch is None else scratch.data_ptr(), size, n), "gated_ffn_forward")
        return out

    def backward(self, dy, x, w_in, w_out, saved, want_dx: bool = True):
        """(dx, dw_in, dw_out); dx is None unless wanted."""
        n = x.shape[0]
        pre, hidden = self._saved(saved, n)
        dx = self._empty(n, self.model) if want_dx else None
        dw_in, dw_out = self._empty(2 * self.hidden, self.model), self._empty(self.model, self.hidden)
        scratch, size = self._scratch(n, 1)
        self._stream()
        _check(self._lib.gated_ffn_backward(
            self.h, self._rows("dy", dy, n), self._stride(dy), self._rows("x", x, n), self._stride(x),
            self._dense("w_in", w_in, (2 * self.hidden, self.model)),
            self._dense("w_out", w_out, (self.model, self.hidden)),
            pre, hidden, None if dx is None else dx.data_ptr(),
            self.model, dw_in.data_ptr(), dw_out.data_ptr(),
            None if scratch is None else scratch.data_ptr(), size, n), "gated_ffn_backward")
        return dx, dw_in, dw_out

    def status(self) -> None:
        """Synchronises; raises if a kernel gave up a wait."""
        gated_ffn_status(self.h)
