"""ctypes binding of liblayer_norm_b200.so: the entry points of include/layer_norm.h, and a
small wrapper that owns the handle, checks tensors and allocates outputs with torch.
No CPU path."""
from __future__ import annotations

import ctypes
import os

from . import build as _build

EXPORTS = ("layer_norm_create", "layer_norm_destroy", "layer_norm_set_stream", "layer_norm_forward",
           "layer_norm_workspace_bytes", "layer_norm_backward", "layer_norm_launch_count", "layer_norm_strerror")

LAYER_NORM_F32, LAYER_NORM_BF16, LAYER_NORM_F16 = 0, 1, 2
MAX_WIDTH = 8192


class LayerNormError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (code %d)" % (where, strerror(code), code))


_lib = None


def load(build_if_missing: bool = False):
    """Load liblayer_norm_b200.so.  Raises if it is missing (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LAYER_NORM_LIB
    if build_if_missing:
        _build.build_one("liblayer_norm_b200.so")
    if not os.path.exists(path):
        raise ImportError("CUDA library %s is not built; run `python -m paper_2603_12145_b200.build`"
                          " (needs nvcc). There is no CPU fallback." % path)
    L = ctypes.CDLL(path)
    vp, i32, i64, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    L.layer_norm_create.argtypes = [ctypes.POINTER(vp), i32, ctypes.c_float, i32]
    L.layer_norm_destroy.argtypes = [vp]
    L.layer_norm_set_stream.argtypes = [vp, vp]
    L.layer_norm_forward.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, i64]
    L.layer_norm_workspace_bytes.argtypes = [vp, i64]
    L.layer_norm_backward.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, vp, vp, size, i64]
    L.layer_norm_launch_count.argtypes = [vp]
    L.layer_norm_strerror.argtypes = [i32]
    for name in EXPORTS:
        getattr(L, name).restype = i32
    L.layer_norm_workspace_bytes.restype = size
    L.layer_norm_launch_count.restype = i64
    L.layer_norm_strerror.restype = ctypes.c_char_p
    _lib = L
    return L


def strerror(code: int) -> str:
    return load().layer_norm_strerror(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise LayerNormError(code, where)


def layer_norm_create(width: int, eps: float, type_: int) -> int:
    h = ctypes.c_void_p()
    _check(load().layer_norm_create(ctypes.byref(h), width, eps, type_), "layer_norm_create")
    return h.value


def layer_norm_destroy(h: int) -> None:
    _check(load().layer_norm_destroy(h), "layer_norm_destroy")


def layer_norm_launch_count(h: int) -> int:
    return int(load().layer_norm_launch_count(h))


# ---- a small owner of the handle ----------------------------------------------------

class LayerNorm:
    """The norm for one width.  Rows are torch CUDA tensors [n, width] of the handle's dtype with a
    contiguous last dimension and any row stride (inputs may have stride 0: one row for all); w and b
    are contiguous float32 [width] or None.  Calls enqueue on the current stream of the device,
    whichever device is current; outputs that are not given are allocated.  One thread at a time.
    A tensor that does not fit raises ValueError, a refusal by the library LayerNormError."""

    def __init__(self, width: int, eps: float = 1e-5, dtype=None, device: str = "cuda:0"):
        import torch
        self.torch = torch
        self.dtype = torch.bfloat16 if dtype is None else dtype
        types = {torch.float32: LAYER_NORM_F32, torch.bfloat16: LAYER_NORM_BF16, torch.float16: LAYER_NORM_F16}
        if self.dtype not in types:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        self.width, self.eps = int(width), float(eps)
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("device must be a CUDA device")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        # the current stream's handle without building a Stream object: a few rows are short
        self._current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
        self._lib = load()
        self._on = None                   # the stream that the handle was last given
        self._sizes = {}                  # workspace bytes by rows
        self._f32 = torch.empty(0, dtype=torch.float32, device=self.device)     # what new buffers are like
        with torch.cuda.device(self.device):
            self.h = layer_norm_create(self.width, self.eps, types[self.dtype])

    def close(self):
        if getattr(self, "h", None):
            layer_norm_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launches(self) -> int:
        return layer_norm_launch_count(self.h)

    def _stream(self):
        stream = self._current(self._index)
        if stream != self._on:
            self._lib.layer_norm_set_stream(self.h, stream)
            self._on = stream

    # -- checks: the library sees pointers only

    def _bad(self, name, v, want):
        raise ValueError("%s must be %s on %s, got %s %s on %s with strides %s"
                         % (name, want, self.device, v.dtype, tuple(v.shape), v.device, v.stride()))

    def _rows(self, name, v, n):
        """The address of [n, width]."""
        if (v.dtype is not self.dtype or v.shape != (n, self.width) or v.get_device() != self._index
                or (self.width > 1 and v.stride(1) != 1)):
            self._bad(name, v, "%s [%d, %d] with a contiguous last dimension" % (self.dtype, n, self.width))
        return v.data_ptr()

    def _dense(self, name, v, shape):
        if v.dtype is not self.torch.float32 or v.shape != shape or v.get_device() != self._index or not v.is_contiguous():
            self._bad(name, v, "contiguous torch.float32 %s" % (shape,))
        return v.data_ptr()

    def _like(self, x):
        """An output [n, width]."""
        if x.is_contiguous():
            return self.torch.empty_like(x)
        return self.torch.empty((x.shape[0], self.width), dtype=self.dtype, device=self.device)

    def _all_rows(self, n, **rows):
        for name, v in rows.items():
            if v is not None:
                self._rows(name, v, n)

    def saved(self, n: int):
        """Buffer in which forward() leaves what backward() needs: float32 [n, 2]."""
        return self._f32.new_empty((n, 2))

    def forward(self, x, w=None, b=None, residual=None, saved=None, out=None, total=None):
        """The normalised rows; with a residual (rows, total): total = x + residual is the stream as it goes on, and
        may be given as x or residual themselves, to be updated in place."""
        dtype, index, width = self.dtype, self._index, self.width
        n = x.shape[0]
        if out is None:
            out = self._like(x)
        row, sx, so, sr, st = (n, width), x.stride(), out.stride(), (0, 1), (0, 1)
        # one look at everything: a few rows are short; what does not fit is named below
        fits = (x.dtype is dtype and out.dtype is dtype and x.shape == row and out.shape == row and x.get_device() == index
                and out.get_device() == index)
        if residual is not None:
            if total is None:
                total = self._like(x)
            sr, st = residual.stride(), total.stride()
            fits = (fits and residual.dtype is dtype and total.dtype is dtype and residual.shape == row and total.shape == row
                    and residual.get_device() == index and total.get_device() == index)
        elif total is not None:
            raise ValueError("total needs a residual")
        if not fits or (width > 1 and not sx[1] == so[1] == sr[1] == st[1] == 1):
            self._all_rows(n, x=x, out=out, residual=residual, total=total)
        shape = (width,)
        self._stream()
        code = self._lib.layer_norm_forward(
            self.h, x.data_ptr(), sx[0], None if residual is None else residual.data_ptr(), sr[0],
            None if w is None else self._dense("w", w, shape), None if b is None else self._dense("b", b, shape),
            None if total is None else total.data_ptr(), st[0], out.data_ptr(), so[0],
            None if saved is None else self._dense("saved", saved, (n, 2)), n)
        if code != 0:
            raise LayerNormError(code, "layer_norm_forward")
        return out if residual is None else (out, total)

    def backward(self, dy, s, w, saved, dsum=None, out=None, want_params: bool = True):
        """(dx, dw, db) for the rows s that were normalised (forward's total, or its x).  dsum: the gradient that
        reaches the stream from behind.  dx is the gradient of x and of the residual alike; dw and db are None unless
        wanted."""
        dtype, index, width = self.dtype, self._index, self.width
        n = s.shape[0]
        dx = self._like(s) if out is None else out
        row, sy, ss, sx, sd = (n, width), dy.stride(), s.stride(), dx.stride(), (0, 1)
        fits = (dy.dtype is dtype and s.dtype is dtype and dx.dtype is dtype and dy.shape == row and s.shape == row
                and dx.shape == row and dy.get_device() == index and s.get_device() == index and dx.get_device() == index)
        if dsum is not None:
            sd = dsum.stride()
            fits = fits and dsum.dtype is dtype and dsum.shape == row and dsum.get_device() == index
        if not fits or (width > 1 and not sy[1] == ss[1] == sx[1] == sd[1] == 1):
            self._all_rows(n, dy=dy, s=s, out=dx, dsum=dsum)
        pw = None if w is None else self._dense("w", w, (width,))
        kept = self._dense("saved", saved, (n, 2))
        dw = db = scratch = None
        size = 0
        if want_params:
            dw, db = self._f32.new_empty(width), self._f32.new_empty(width)
            if n not in self._sizes:
                if len(self._sizes) > 1000:
                    self._sizes.clear()
                self._sizes[n] = self._lib.layer_norm_workspace_bytes(self.h, n)
            size = self._sizes[n]
            scratch = self._f32.new_empty(size // 4)
        self._stream()
        code = self._lib.layer_norm_backward(
            self.h, dy.data_ptr(), sy[0], s.data_ptr(), ss[0], pw, kept, None if dsum is None else dsum.data_ptr(), sd[0],
            dx.data_ptr(), sx[0], None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(),
            None if scratch is None else scratch.data_ptr(), size, n)
        if code != 0:
            raise LayerNormError(code, "layer_norm_backward")
        return dx, dw, db
