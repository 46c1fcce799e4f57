"""ctypes binding of libgated_recurrence_b200.so: the entry points of include/gated_recurrence.h,
and a small wrapper that owns the handle, checks tensors and allocates outputs with torch.
No CPU path."""
from __future__ import annotations

import ctypes
import os
import struct

from . import build as _build

EXPORTS = ("gated_recurrence_create", "gated_recurrence_destroy", "gated_recurrence_set_stream",
           "gated_recurrence_saved_bytes", "gated_recurrence_workspace_bytes", "gated_recurrence_forward",
           "gated_recurrence_backward", "gated_recurrence_step", "gated_recurrence_launch_count",
           "gated_recurrence_strerror")

GATED_RECURRENCE_F32, GATED_RECURRENCE_BF16, GATED_RECURRENCE_F16 = 0, 1, 2


class GatedRecurrenceError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (code %d)" % (where, strerror(code), code))


class Seq(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_t", ctypes.c_int64)]


class Args(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("time", ctypes.c_int64), ("x", Seq), ("r", Seq), ("i", Seq),
                ("reset", Seq), ("a", ctypes.c_void_p), ("state", ctypes.c_void_p), ("state_out", ctypes.c_void_p),
                ("y", Seq), ("saved", ctypes.c_void_p), ("dy", Seq), ("dstate_out", ctypes.c_void_p), ("dx", Seq),
                ("dr", Seq), ("di", Seq), ("da", ctypes.c_void_p), ("dstate", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


_PACKED = struct.Struct("=%dq" % (ctypes.sizeof(Args) // 8))      # all fields of Args, one after the other
_NONE = (0, 0, 0)
_lib = None


def load(build_if_missing: bool = False):
    """Load libgated_recurrence_b200.so.  Raises if it is missing (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.GATED_RECURRENCE_LIB
    if build_if_missing:
        _build.build_one("libgated_recurrence_b200.so")
    if not os.path.exists(path):
        raise ImportError("CUDA library %s is not built; run `python -m paper_2603_12145_b200.build`"
                          " (needs nvcc). There is no CPU fallback." % path)
    L = ctypes.CDLL(path)
    vp, i32, i64, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    L.gated_recurrence_create.argtypes = [ctypes.POINTER(vp), i32, i32]
    L.gated_recurrence_destroy.argtypes = [vp]
    L.gated_recurrence_set_stream.argtypes = [vp, vp]
    L.gated_recurrence_saved_bytes.argtypes = [vp, i64, i64]
    L.gated_recurrence_workspace_bytes.argtypes = [vp, i64, i64, i32]
    L.gated_recurrence_forward.argtypes = [vp, vp]
    L.gated_recurrence_backward.argtypes = [vp, vp]
    L.gated_recurrence_step.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, i64]
    L.gated_recurrence_launch_count.argtypes = [vp]
    L.gated_recurrence_strerror.argtypes = [i32]
    for name in EXPORTS:
        getattr(L, name).restype = i32
    L.gated_recurrence_saved_bytes.restype = size
    L.gated_recurrence_workspace_bytes.restype = size
    L.gated_recurrence_launch_count.restype = i64
    L.gated_recurrence_strerror.restype = ctypes.c_char_p
    _lib = L
    return L


def strerror(code: int) -> str:
    return load().gated_recurrence_strerror(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise GatedRecurrenceError(code, where)


def gated_recurrence_create(channels: int, type_: int) -> int:
    h = ctypes.c_void_p()
    _check(load().gated_recurrence_create(ctypes.byref(h), channels, type_), "gated_recurrence_create")
    return h.value


def gated_recurrence_destroy(h: int) -> None:
    _check(load().gated_recurrence_destroy(h), "gated_recurrence_destroy")


def gated_recurrence_launch_count(h: int) -> int:
    return int(load().gated_recurrence_launch_count(h))


# ---- a small owner of the handle ----------------------------------------------------

class GatedRecurrence:
    """The recurrence for one layer's channels.

    Sequences are torch CUDA tensors [batch, time, channels] of the handle's dtype with any
    strides but a contiguous last dimension (a time-major rollout is `v.transpose(0, 1)`);
    single tokens are [n, channels].  reset / done are uint8 or bool [batch, time] / [n].
    a [channels] (<= 0) and states [n, channels] are contiguous float32.  Calls enqueue on the
    current stream of the device, whichever device is current; outputs that are not given are
    allocated.  One thread at a time.  A tensor that does not fit raises ValueError, a refusal
    by the library GatedRecurrenceError."""

    def __init__(self, channels: int, dtype=None, device: str = "cuda:0"):
        import torch
        self.torch = torch
        self.dtype = torch.bfloat16 if dtype is None else dtype
        types = {torch.float32: GATED_RECURRENCE_F32, torch.bfloat16: GATED_RECURRENCE_BF16,
                 torch.float16: GATED_RECURRENCE_F16}
        if self.dtype not in types:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        self.channels = int(channels)
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
        self._sizes = {}                  # bytes of saved and workspaces by shape
        self._f32 = torch.empty(0, dtype=torch.float32, device=self.device)     # what new buffers are like
        with torch.cuda.device(self.device):
            self.h = gated_recurrence_create(self.channels, types[self.dtype])

    def close(self):
        if getattr(self, "h", None):
            gated_recurrence_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launches(self) -> int:
        return gated_recurrence_launch_count(self.h)

    def _stream(self):
        stream = self._current(self._index)
        if stream != self._on:
            self._lib.gated_recurrence_set_stream(self.h, stream)
            self._on = stream

    # -- checks: the library sees pointers only

    def _bad(self, name, v, want):
        raise ValueError("%s must be %s on %s, got %s %s on %s with strides %s"
                         % (name, want, self.device, v.dtype, tuple(v.shape), v.device, v.stride()))

    def _seq(self, name, v, shape):
        """(address, stride of the batch, stride of time)."""
        s = v.stride()
        if (v.dtype is not self.dtype or v.shape != shape or v.get_device() != self._index
                or (s[2] != 1 and self.channels > 1)):
            self._bad(name, v, "%s %s with a contiguous last dimension" % (self.dtype, list(shape)))
        return v.data_ptr(), s[0], s[1]

    def _mask(self, name, v, shape):
        if v.dtype not in (self.torch.uint8, self.torch.bool) or v.shape != shape or v.get_device() != self._index:
            self._bad(name, v, "uint8 or bool %s" % (shape,))
        return v

    def _row(self, name, v, n):
        if (v.dtype is not self.dtype or v.shape != (n, self.channels) or v.get_device() != self._index
                or (self.channels > 1 and v.stride(1) != 1)):
            self._bad(name, v, "%s [%d, %d] with a contiguous last dimension" % (self.dtype, n, self.channels))

    def _dense(self, name, v, shape):
        if v.dtype is not self.torch.float32 or v.shape != shape or v.get_device() != self._index or not v.is_contiguous():
            self._bad(name, v, "contiguous torch.float32 %s" % (shape,))
        return v.data_ptr()

    def _like(self, v):
        """An output [batch, time, channels] with the order of v's dimensions."""
        out = self.torch.empty_like(v)               # keeps the order of what is dense
        if out.stride(2) != 1 and self.channels > 1:                     # (of overlapping rows the channels' place too)
            out = self.torch.empty(v.shape, dtype=self.dtype, device=self.device)
        if out.stride(0) > out.stride(1) and v.stride(0) < v.stride(1):
            b, t = v.shape[0], v.shape[1]
            return self.torch.empty((t, b, self.channels), dtype=self.dtype, device=self.device).transpose(0, 1)
        return out

    # -- buffers

    def state(self, n: int):
        """Buffer for the recurrent state, float32 [n, channels]."""
        return self._f32.new_empty((n, self.channels))

    def _size(self, batch, time, what):
        """Bytes of `saved` ("saved"), of the forward (0) and of the backward workspace (1)."""
        key = (batch, time, what)
        if key not in self._sizes:
            if len(self._sizes) > 1000:
                self._sizes.clear()
            self._sizes[key] = (self._lib.gated_recurrence_saved_bytes(self.h, batch, time) if what == "saved" else
                                self._lib.gated_recurrence_workspace_bytes(self.h, batch, time, what))
        return self._sizes[key]

    def saved(self, batch: int, time: int):
        """Buffer in which sequence() leaves what backward() needs."""
        return self._f32.new_empty(self._size(batch, time, "saved") // 4)

    # -- sequences

    def _common(self, x, r, i, a, reset):
        """The shape, and the packed arguments that both passes begin with."""
        shape = x.shape
        if len(shape) != 3 or shape[2] != self.channels:
            self._bad("x", x, "%s [batch, time, %d]" % (self.dtype, self.channels))
        mask = _NONE
        if reset is not None:
            self._mask("reset", reset, shape[:2])
            mask = (reset.data_ptr(),) + reset.stride()
        return shape, (shape[0], shape[1], *self._seq("x", x, shape), *self._seq("r", r, shape), *self._seq("i", i, shape),
                       *mask, self._dense("a", a, (self.channels,)))

    def _call(self, call, where, *fields):
        code = call(self.h, _PACKED.pack(*fields))
        if code != 0:
            raise GatedRecurrenceError(code, where)

    def sequence(self, x, r, i, a, reset=None, state=None, state_out=None, saved=None, out=None):
        """y of the recurrence.  saved (from saved()) is filled for backward()."""
        shape, first = self._common(x, r, i, a, reset)
        n, t = shape[0], shape[1]
        if out is None:
            out = self._like(x)
        states = (n, self.channels)
        size = self._size(n, t, 0)
        scratch = self._f32.new_empty(size // 4) if size else None
        self._stream()
        self._call(self._lib.gated_recurrence_forward, "gated_recurrence_forward", *first,
                   0 if state is None else self._dense("state", state, states),
                   0 if state_out is None else self._dense("state_out", state_out, states), *self._seq("out", out, shape),
                   0 if saved is None else self._dense("saved", saved, (self._size(n, t, "saved") // 4,)),
                   *_NONE, 0, *_NONE, *_NONE, *_NONE, 0, 0, scratch.data_ptr() if size else 0, size)
        return out

    def backward(self, dy, x, r, i, a, saved, reset=None, dstate_out=None, want_dstate=False):
        """Gradients as a dict: dx, dr, di, da, dstate (None where not wanted).  dstate_out: gradient of the state that
        sequence() returned."""
        shape, first = self._common(x, r, i, a, reset)
        n, t = shape[0], shape[1]
        states = (n, self.channels)
        dx, dr, di, da = self._like(x), self._like(r), self._like(i), self.torch.empty_like(a)
        dstate = self.state(n) if want_dstate else None
        size = self._size(n, t, 1)
        scratch = self._f32.new_empty(size // 4) if size else None
        self._stream()
        self._call(self._lib.gated_recurrence_backward, "gated_recurrence_backward", *first, 0, 0, *_NONE,
                   self._dense("saved", saved, (self._size(n, t, "saved") // 4,)), *self._seq("dy", dy, shape),
                   0 if dstate_out is None else self._dense("dstate_out", dstate_out, states), dx.data_ptr(), *dx.stride()[:2],
                   dr.data_ptr(), *dr.stride()[:2], di.data_ptr(), *di.stride()[:2], da.data_ptr(),
                   0 if dstate is None else dstate.data_ptr(), scratch.data_ptr() if size else 0, size)
        return {"dx": dx, "dr": dr, "di": di, "da": da, "dstate": dstate}

    # -- single tokens

    def step(self, x, r, i, a, state, done=None, state_out=None, out=None):
        """One token of n rows; the state is updated in place unless state_out is given."""
        t, index, dtype, ch = self.torch, self._index, self.dtype, self.channels
        n = x.shape[0]
        if out is None:
            out = t.empty_like(x) if x.is_contiguous() else t.empty((n, ch), dtype=dtype, device=self.device)
        if state_out is None:
            state_out = state
        row, f32 = (n, ch), t.float32
        sx, sr, si, so = x.stride(), r.stride(), i.stride(), out.stride()
        # one look at everything: a single token is short; what does not fit is named below
        if not (x.dtype is dtype and r.dtype is dtype and i.dtype is dtype and out.dtype is dtype and a.dtype is f32
                and state.dtype is f32 and state_out.dtype is f32 and x.shape == row and r.shape == row and i.shape == row
                and out.shape == row and state.shape == row and state_out.shape == row and a.shape == (ch,)
                and x.get_device() == index and r.get_device() == index and i.get_device() == index
                and out.get_device() == index and a.get_device() == index and state.get_device() == index
                and state_out.get_device() == index and sx[1] == 1 and sr[1] == 1 and si[1] == 1 and so[1] == 1
                and a.is_contiguous() and state.is_contiguous() and state_out.is_contiguous()):
            for name, v in (("x", x), ("r", r), ("i", i), ("out", out)):
                self._row(name, v, n)
            for name, v, want in (("a", a, (ch,)), ("state", state, row), ("state_out", state_out, row)):
                self._dense(name, v, want)
        if done is not None:
            self._mask("done", done, (n,))
        self._stream()
        code = self._lib.gated_recurrence_step(
            self.h, x.data_ptr(), sx[0], r.data_ptr(), sr[0], i.data_ptr(), si[0],
            None if done is None else done.data_ptr(), 0 if done is None else done.stride(0), a.data_ptr(),
            state.data_ptr(), state_out.data_ptr(), out.data_ptr(), so[0], n)
        if code != 0:
            raise GatedRecurrenceError(code, "gated_recurrence_step")
        return out
