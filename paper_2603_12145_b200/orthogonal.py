"""ctypes binding of liborthogonal_b200.so: the entry points of include/orthogonal.h, and a small
wrapper that owns the handle, checks tensors and allocates outputs with torch.
No CPU path."""
from __future__ import annotations

import ctypes
import os

from . import build as _build

EXPORTS = ("orthogonal_create", "orthogonal_destroy", "orthogonal_set_stream", "orthogonal_workspace_bytes",
           "orthogonal_update", "orthogonal_status", "orthogonal_launch_count", "orthogonal_strerror")

ORTHOGONAL_F32, ORTHOGONAL_BF16, ORTHOGONAL_F16 = 0, 1, 2
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


class OrthogonalError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (code %d)" % (where, strerror(code), code))


_lib = None


def load(build_if_missing: bool = False):
    """Load liborthogonal_b200.so.  Raises if it is missing (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.ORTHOGONAL_LIB
    if build_if_missing:
        _build.build_one("liborthogonal_b200.so")
    if not os.path.exists(path):
        raise ImportError("CUDA library %s is not built; run `python -m paper_2603_12145_b200.build`"
                          " (needs nvcc). There is no CPU fallback." % path)
    L = ctypes.CDLL(path)
    vp, i32, i64, size, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
    L.orthogonal_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32, f32, f32, f32, f32, i32]
    L.orthogonal_destroy.argtypes = [vp]
    L.orthogonal_set_stream.argtypes = [vp, vp]
    L.orthogonal_workspace_bytes.argtypes = [vp, i64]
    L.orthogonal_update.argtypes = [vp, vp, i64, i64, vp, i64, i64, vp, size, i64]
    L.orthogonal_status.argtypes = [vp]
    L.orthogonal_launch_count.argtypes = [vp]
    L.orthogonal_strerror.argtypes = [i32]
    for name in EXPORTS:
        getattr(L, name).restype = i32
    L.orthogonal_workspace_bytes.restype = size
    L.orthogonal_launch_count.restype = i64
    L.orthogonal_strerror.restype = ctypes.c_char_p
    _lib = L
    return L


def strerror(code: int) -> str:
    return load().orthogonal_strerror(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise OrthogonalError(code, where)


def orthogonal_create(rows: int, cols: int, steps: int, a: float, b: float, c: float, eps: float, type_: int) -> int:
    h = ctypes.c_void_p()
    _check(load().orthogonal_create(ctypes.byref(h), rows, cols, steps, a, b, c, eps, type_), "orthogonal_create")
    return h.value


def orthogonal_destroy(h: int) -> None:
    _check(load().orthogonal_destroy(h), "orthogonal_destroy")


def orthogonal_status(h: int) -> None:
    _check(load().orthogonal_status(h), "orthogonal_status")


def orthogonal_launch_count(h: int) -> int:
    return int(load().orthogonal_launch_count(h))


# ---- a small owner of the handle ----------------------------------------------------

class Orthogonal:
    """The update for one matrix size.  G is a torch CUDA tensor [rows, cols] or [batch, rows, cols] of
    the handle's dtype with a contiguous last dimension and any other strides; the update has its shape,
    in bfloat16.  Calls enqueue on the current stream of the device, whichever device is current; an
    output that is not given is allocated.  One thread at a time.  A tensor that does not fit raises
    ValueError, a refusal by the library OrthogonalError."""

    def __init__(self, rows: int, cols: int, dtype=None, steps: int = 5, coefficients=COEFFICIENTS, eps: float = 1e-7,
                 device: str = "cuda:0"):
        import torch
        self.torch = torch
        self.dtype = torch.bfloat16 if dtype is None else dtype
        types = {torch.float32: ORTHOGONAL_F32, torch.bfloat16: ORTHOGONAL_BF16, torch.float16: ORTHOGONAL_F16}
        if self.dtype not in types:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        a, b, c = coefficients
        self.rows, self.cols, self.steps, self.coefficients, self.eps = int(rows), int(cols), int(steps), (a, b, c), float(eps)
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("device must be a CUDA device")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        # the current stream's handle without building a Stream object
        self._current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
        self._lib = load()
        self._on = None                   # the stream that the handle was last given
        self._f32 = torch.empty(0, dtype=torch.float32, device=self.device)     # what new buffers are like
        with torch.cuda.device(self.device):
            self.h = orthogonal_create(self.rows, self.cols, self.steps, a, b, c, self.eps, types[self.dtype])

    def close(self):
        if getattr(self, "h", None):
            with self.torch.cuda.device(self.device):
                orthogonal_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launches(self) -> int:
        return orthogonal_launch_count(self.h)

    def _stream(self):
        stream = self._current(self._index)
        if stream != self._on:
            self._lib.orthogonal_set_stream(self.h, stream)
            self._on = stream

    def _matrices(self, name, v, dtype, shape):
        """(address, stride of the batch, stride of the rows)."""
        strides = v.stride()
        if v.dtype is not dtype or v.shape != shape or v.get_device() != self._index or (self.cols > 1 and strides[-1] != 1):
            raise ValueError("%s must be %s %s on %s with a contiguous last dimension, got %s %s on %s with strides %s"
                             % (name, dtype, tuple(shape), self.device, v.dtype, tuple(v.shape), v.device, strides))
        return v.data_ptr(), strides[0] if len(shape) == 3 else 0, strides[-2]

    def update(self, g, out=None):
        """The orthogonalised update of g, each matrix of a batch by itself."""
        t = self.torch
        if g.dim() not in (2, 3):
            raise ValueError("g must be [rows, cols] or [batch, rows, cols], got %s" % (tuple(g.shape),))
        batch = g.shape[0] if g.dim() == 3 else 1
        shape = (batch, self.rows, self.cols) if g.dim() == 3 else (self.rows, self.cols)
        pg, gb, gr = self._matrices("g", g, self.dtype, shape)
        if out is None:
            out = t.empty(shape, dtype=t.bfloat16, device=self.device)
        po, ob, orow = self._matrices("out", out, t.bfloat16, shape)
        size = self._lib.orthogonal_workspace_bytes(self.h, batch)
        scratch = self._f32.new_empty(size // 4) if size else None
        self._stream()
        code = self._lib.orthogonal_update(self.h, pg, gb, gr, po, ob, orow, None if scratch is None else scratch.data_ptr(),
                                           size, batch)
        if code != 0:
            raise OrthogonalError(code, "orthogonal_update")
        return out

    def status(self) -> None:
        """Synchronises; raises if a kernel gave up a wait."""
        orthogonal_status(self.h)
