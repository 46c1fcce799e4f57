"""ctypes binding of libssm_b200.so: the entry points of include/ssm.h, and a small
wrapper that owns the handle, checks tensors and allocates outputs with torch.
No CPU path."""
from __future__ import annotations

import ctypes
import os

from . import build as _build

EXPORTS = ("ssm_create", "ssm_destroy", "ssm_set_stream", "ssm_conv_workspace_bytes", "ssm_conv_forward",
           "ssm_conv_backward", "ssm_conv_step", "ssm_scan_saved_bytes", "ssm_scan_workspace_bytes",
           "ssm_scan_forward", "ssm_scan_backward", "ssm_scan_step", "ssm_launch_count", "ssm_strerror")

SSM_F32, SSM_BF16, SSM_F16 = 0, 1, 2
MAX_STATES, MAX_WIDTH = 64, 4


class SsmError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (code %d)" % (where, strerror(code), code))


class Seq(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_t", ctypes.c_int64)]


class ConvArgs(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("time", ctypes.c_int64), ("x", Seq), ("reset", Seq),
                ("w", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("history", ctypes.c_void_p), ("y", Seq),
                ("history_out", ctypes.c_void_p), ("dy", Seq), ("dx", Seq), ("dw", ctypes.c_void_p),
                ("dbias", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class ScanArgs(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("time", ctypes.c_int64), ("x", Seq), ("dt", Seq), ("z", Seq),
                ("b", Seq), ("c", Seq), ("reset", Seq), ("a", ctypes.c_void_p), ("d", ctypes.c_void_p),
                ("dt_bias", ctypes.c_void_p), ("state", ctypes.c_void_p), ("state_out", ctypes.c_void_p),
                ("y", Seq), ("saved", ctypes.c_void_p), ("dy", Seq), ("dstate_out", ctypes.c_void_p),
                ("dx", Seq), ("ddt", Seq), ("dz", Seq), ("db", Seq), ("dc", Seq), ("da", ctypes.c_void_p),
                ("dd", ctypes.c_void_p), ("ddt_bias", ctypes.c_void_p), ("dstate", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


_lib = None


def load(build_if_missing: bool = False):
    """Load libssm_b200.so.  Raises if it is missing (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.SSM_LIB
    if build_if_missing:
        _build.build_one("libssm_b200.so")
    if not os.path.exists(path):
        raise ImportError("CUDA library %s is not built; run `python -m paper_2603_12145_b200.build`"
                          " (needs nvcc). There is no CPU fallback." % path)
    L = ctypes.CDLL(path)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    L.ssm_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32, i32, i32]
    L.ssm_destroy.argtypes = [vp]
    L.ssm_set_stream.argtypes = [vp, vp]
    L.ssm_conv_workspace_bytes.argtypes = [vp, i64, i64]
    L.ssm_conv_forward.argtypes = [vp, vp]
    L.ssm_conv_backward.argtypes = [vp, vp]
    L.ssm_conv_step.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, i64]
    L.ssm_scan_saved_bytes.argtypes = [vp, i64, i64]
    L.ssm_scan_workspace_bytes.argtypes = [vp, i64, i64, i32]
    L.ssm_scan_forward.argtypes = [vp, vp]
    L.ssm_scan_backward.argtypes = [vp, vp]
    L.ssm_scan_step.argtypes = [vp] + [vp, i64] * 6 + [vp] * 6 + [i64, i64]
    L.ssm_launch_count.argtypes = [vp]
    L.ssm_strerror.argtypes = [i32]
    for name in EXPORTS:
        getattr(L, name).restype = i32
    for name in ("ssm_conv_workspace_bytes", "ssm_scan_saved_bytes", "ssm_scan_workspace_bytes"):
        getattr(L, name).restype = ctypes.c_size_t
    L.ssm_launch_count.restype = i64
    L.ssm_strerror.restype = ctypes.c_char_p
    _lib = L
    return L


def strerror(code: int) -> str:
    return load().ssm_strerror(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise SsmError(code, where)


def ssm_create(channels: int, states: int, groups: int, width: int, type_: int) -> int:
    h = ctypes.c_void_p()
    _check(load().ssm_create(ctypes.byref(h), channels, states, groups, width, type_), "ssm_create")
    return h.value


def ssm_destroy(h: int) -> None:
    _check(load().ssm_destroy(h), "ssm_destroy")


def ssm_launch_count(h: int) -> int:
    return int(load().ssm_launch_count(h))


# ---- a small owner of the handle ----------------------------------------------------

class Ssm:
    """The convolution and the scan for one layer's sizes.

    Sequences are torch CUDA tensors [batch, time, features] of the handle's dtype with any
    strides but a contiguous last dimension (a time-major rollout is `v.transpose(0, 1)`);
    single tokens are [n, features].  reset / done are uint8 or bool [batch, time] / [n].
    Parameters and recurrent states are contiguous float32.  Calls enqueue on the current
    stream of the device, whichever device is current; outputs that are not given are
    allocated.  One thread at a time.  A tensor that does not fit raises ValueError, a refusal
    by the library SsmError."""

    def __init__(self, channels: int, states: int = 16, groups: int = 1, width: int = 4, dtype=None,
                 device: str = "cuda:0"):
        import torch
        self.torch = torch
        self.dtype = torch.bfloat16 if dtype is None else dtype
        types = {torch.float32: SSM_F32, torch.bfloat16: SSM_BF16, torch.float16: SSM_F16}
        if self.dtype not in types:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        self.channels, self.states, self.groups, self.width = int(channels), int(states), int(groups), int(width)
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
            self.h = ssm_create(self.channels, self.states, self.groups, self.width, types[self.dtype])

    def close(self):
        if getattr(self, "h", None):
            ssm_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launches(self) -> int:
        return ssm_launch_count(self.h)

    def _stream(self):
        stream = self._current(self._index)
        if stream != self._on:
            self._lib.ssm_set_stream(self.h, stream)
            self._on = stream

    # -- checks: the library sees pointers only

    def _bad(self, name, v, want):
        raise ValueError("%s must be %s on %s, got %s %s on %s with strides %s"
                         % (name, want, self.device, v.dtype, tuple(v.shape), v.device, v.stride()))

    def _seq(self, name, v, batch, time, features):
        if (v.dtype is not self.dtype or v.shape != (batch, time, features) or v.get_device() != self._index
                or (features > 1 and v.stride(2) != 1)):
            self._bad(name, v, "%s [%d, %d, %d] with a contiguous last dimension" % (self.dtype, batch, time, features))
        return Seq(v.data_ptr(), v.stride(0), v.stride(1))

    def _mask(self, name, v, shape):
        if v.dtype not in (self.torch.uint8, self.torch.bool) or v.shape != shape or v.get_device() != self._index:
            self._bad(name, v, "uint8 or bool %s" % (shape,))
        return v

    def _row(self, name, v, n, features):
        if (v.dtype is not self.dtype or v.shape != (n, features) or v.get_device() != self._index
                or (features > 1 and v.stride(1) != 1)):
            self._bad(name, v, "%s [%d, %d] with a contiguous last dimension" % (self.dtype, n, features))
        return v.data_ptr()

    def _dense(self, name, v, shape, dtype=None):
        dtype = self.torch.float32 if dtype is None else dtype
        if v.dtype is not dtype or v.shape != shape or v.get_device() != self._index or not v.is_contiguous():
            self._bad(name, v, "contiguous %s %s" % (dtype, shape))
        return v.data_ptr()

    def _like(self, v, features):
        """An output [batch, time, features] with the order of v's dimensions."""
        b, t = v.shape[0], v.shape[1]
        if v.stride(0) < v.stride(1):
            return self.torch.empty((t, b, features), dtype=self.dtype, device=self.device).transpose(0, 1)
        return self.torch.empty((b, t, features), dtype=self.dtype, device=self.device)

    def _f32(self, *shape):
        return self.torch.empty(shape, dtype=self.torch.float32, device=self.device)

    # -- buffers

    def history(self, n: int):
        """Buffer for the convolution's last inputs, [n, width - 1, channels]."""
        return self.torch.empty((n, self.width - 1, self.channels), dtype=self.dtype, device=self.device)

    def state(self, n: int):
        """Buffer for the recurrent state, float32 [n, channels, states]."""
        return self._f32(n, self.channels, self.states)

    def saved(self, batch: int, time: int):
        """Buffer in which scan() leaves what scan_backward() needs."""
        return self._f32(int(self._lib.ssm_scan_saved_bytes(self.h, batch, time)) // 4)

    def _scratch(self, size):
        return self.torch.empty((size,), dtype=self.torch.uint8, device=self.device) if size else None

    # -- convolution

    def _conv_args(self, x, w, bias, reset, history):
        b, t, d = x.shape
        a = ConvArgs(batch=b, time=t, x=self._seq("x", x, b, t, self.channels),
                     w=self._dense("w", w, (d, self.width)))
        if bias is not None:
            a.bias = self._dense("bias", bias, (d,))
        if reset is not None:
            self._mask("reset", reset, (b, t))
            a.reset = Seq(reset.data_ptr(), reset.stride(0), reset.stride(1))
        if history is not None:
            a.history = self._dense("history", history, (b, self.width - 1, d), self.dtype)
        return a

    def conv(self, x, w, bias=None, reset=None, history=None, history_out=None, out=None):
        """y = silu(causal convolution of x).  w float32 [channels, width], oldest tap first."""
        a = self._conv_args(x, w, bias, reset, history)
        if out is None:
            out = self._like(x, self.channels)
        a.y = self._seq("out", out, a.batch, a.time, self.channels)
        if history_out is not None:
            a.history_out = self._dense("history_out", history_out, (a.batch, self.width - 1, self.channels),
                                        self.dtype)
        self._stream()
        _check(self._lib.ssm_conv_forward(self.h, ctypes.byref(a)), "ssm_conv_forward")
        return out

    def conv_backward(self, dy, x, w, bias=None, reset=None, history=None):
        """(dx, dw, dbias); dbias is None without a bias.  The history is a constant."""
        a = self._conv_args(x, w, bias, reset, history)
        dx = self._like(x, self.channels)
        dw = self._f32(self.channels, self.width)
        dbias = self._f32(self.channels) if bias is not None else None
        scratch = self._scratch(self._lib.ssm_conv_workspace_bytes(self.h, a.batch, a.time))
        a.dy = self._seq("dy", dy, a.batch, a.time, self.channels)
        a.dx = self._seq("dx", dx, a.batch, a.time, self.channels)
        a.dw = dw.data_ptr()
        if dbias is not None:
            a.dbias = dbias.data_ptr()
        if scratch is not None:
            a.workspace, a.workspace_bytes = scratch.data_ptr(), scratch.numel()
        self._stream()
        _check(self._lib.ssm_conv_backward(self.h, ctypes.byref(a)), "ssm_conv_backward")
        return dx, dw, dbias

    def conv_step(self, x, history, w, bias=None, done=None, history_out=None, out=None):
        """One token of n rows; the history is updated in place unless history_out is given."""
        t, index, dtype, d = self.torch, self._index, self.dtype, self.channels
        n = x.shape[0]
        if out is None:
            out = t.empty((n, d), dtype=dtype, device=self.device)
        if history_out is None:
            history_out = history
        row, shape, sx, so = (n, d), (n, self.width - 1, d), x.stride(), out.stride()
        # one look at everything: a single token is short; what does not fit is named below
        if not (x.dtype is dtype and out.dtype is dtype and history.dtype is dtype and history_out.dtype is dtype
                and w.dtype is t.float32 and x.shape == row and out.shape == row and history.shape == shape
                and history_out.shape == shape and w.shape == (d, self.width) and x.get_device() == index
                and out.get_device() == index and history.get_device() == index and history_out.get_device() == index
                and w.get_device() == index and sx[1] == 1 and so[1] == 1 and history.is_contiguous()
                and history_out.is_contiguous() and w.is_contiguous()):
            self._row("x", x, n, d)
            self._row("out", out, n, d)
            self._dense("w", w, (d, self.width))
            self._dense("history", history, shape, dtype)
            self._dense("history_out", history_out, shape, dtype)
        if done is not None:
            self._mask("done", done, (n,))
        self._stream()
        code = self._lib.ssm_conv_step(
            self.h, x.data_ptr(), sx[0], None if done is None else done.data_ptr(), 0 if done is None else done.stride(0),
            w.data_ptr(), None if bias is None else self._dense("bias", bias, (d,)), history.data_ptr(),
            history_out.data_ptr(), out.data_ptr(), so[0], n)
        if code != 0:
            raise SsmError(code, "ssm_conv_step")
        return out

    # -- scan

    def _scan_args(self, x, dt, a, b, c, d, z, dt_bias, reset, state):
        n, t, ch = x.shape[0], x.shape[1], self.channels
        narrow = self.groups * self.states
        args = ScanArgs(batch=n, time=t, x=self._seq("x", x, n, t, ch), dt=self._seq("dt", dt, n, t, ch),
                        b=self._seq("b", b, n, t, narrow), c=self._seq("c", c, n, t, narrow),
                        a=self._dense("a", a, (ch, self.states)))
        if z is not None:
            args.z = self._seq("z", z, n, t, ch)
        if d is not None:
            args.d = self._dense("d", d, (ch,))
        if dt_bias is not None:
            args.dt_bias = self._dense("dt_bias", dt_bias, (ch,))
        if reset is not None:
            self._mask("reset", reset, (n, t))
            args.reset = Seq(reset.data_ptr(), reset.stride(0), reset.stride(1))
        if state is not None:
            args.state = self._dense("state", state, (n, ch, self.states))
        return args

    def _workspace(self, args, backward):
        scratch = self._scratch(self._lib.ssm_scan_workspace_bytes(self.h, args.batch, args.time, backward))
        if scratch is not None:
            args.workspace, args.workspace_bytes = scratch.data_ptr(), scratch.numel()
        return scratch

    def scan(self, x, dt, a, b, c, d=None, z=None, dt_bias=None, reset=None, state=None, state_out=None,
             saved=None, out=None):
        """y of the scan.  b, c [batch, time, groups * states]; a float32 [channels, states]; saved (from
        saved()) is filled for scan_backward()."""
        args = self._scan_args(x, dt, a, b, c, d, z, dt_bias, reset, state)
        if out is None:
            out = self._like(x, self.channels)
        args.y = self._seq("out", out, args.batch, args.time, self.channels)
        if state_out is not None:
            args.state_out = self._dense("state_out", state_out, (args.batch, self.channels, self.states))
        if saved is not None:
            args.saved = self._saved(saved, args)
        scratch = self._workspace(args, 0)
        self._stream()
        _check(self._lib.ssm_scan_forward(self.h, ctypes.byref(args)), "ssm_scan_forward")
        del scratch
        return out

    def _saved(self, saved, args):
        need = int(self._lib.ssm_scan_saved_bytes(self.h, args.batch, args.time)) // 4
        return self._dense("saved", saved, (need,))

    def scan_backward(self, dy, x, dt, a, b, c, saved, d=None, z=None, dt_bias=None, reset=None,
                      dstate_out=None, want_dstate=False):
        """Gradients as a dict: dx, ddt, da, db, dc, dd, dz, ddt_bias, dstate (None where the input
        is absent or not wanted).  dstate_out: gradient of the state that scan() returned."""
        args = self._scan_args(x, dt, a, b, c, d, z, dt_bias, reset, None)
        n, t, ch, narrow = args.batch, args.time, self.channels, self.groups * self.states
        out = {"dx": self._like(x, ch), "ddt": self._like(dt, ch), "da": self._f32(ch, self.states),
               "db": self._like(b, narrow), "dc": self._like(c, narrow),
               "dd": self._f32(ch) if d is not None else None, "dz": self._like(z, ch) if z is not None else None,
               "ddt_bias": self._f32(ch) if dt_bias is not None else None,
               "dstate": self.state(n) if want_dstate else None}
        args.dy = self._seq("dy", dy, n, t, ch)
        args.saved = self._saved(saved, args)
        for key, features in (("dx", ch), ("ddt", ch), ("dz", ch), ("db", narrow), ("dc", narrow)):
            if out[key] is not None:
                setattr(args, key, self._seq(key, out[key], n, t, features))
        for key in ("da", "dd", "ddt_bias", "dstate"):
            if out[key] is not None:
                setattr(args, key, out[key].data_ptr())
        if dstate_out is not None:
            args.dstate_out = self._dense("dstate_out", dstate_out, (n, ch, self.states))
        scratch = self._workspace(args, 1)
        self._stream()
        _check(self._lib.ssm_scan_backward(self.h, ctypes.byref(args)), "ssm_scan_backward")
        del scratch
        return out

    def scan_step(self, x, dt, a, b, c, state, d=None, z=None, dt_bias=None, done=None, state_out=None, out=None):
        """One token of n rows; the state is updated in place unless state_out is given."""
        t, index, dtype, ch = self.torch, self._index, self.dtype, self.channels
        n, narrow = x.shape[0], self.groups * self.states
        if out is None:
            out = t.empty((n, ch), dtype=dtype, device=self.device)
        if state_out is None:
            state_out = state
        row, thin, shape, rates, f32 = (n, ch), (n, narrow), (n, ch, self.states), (ch, self.states), t.float32
        sx, sdt, sb, sc, so = x.stride(), dt.stride(), b.stride(), c.stride(), out.stride()
        # one look at everything: a single token is short; what does not fit is named below
        if not (x.dtype is dtype and dt.dtype is dtype and b.dtype is dtype and c.dtype is dtype and out.dtype is dtype
                and a.dtype is f32 and state.dtype is f32 and state_out.dtype is f32
                and x.shape == row and dt.shape == row and out.shape == row and b.shape == thin and c.shape == thin
                and a.shape == rates and state.shape == shape and state_out.shape == shape
                and x.get_device() == index and dt.get_device() == index and b.get_device() == index
                and c.get_device() == index and out.get_device() == index and a.get_device() == index
                and state.get_device() == index and state_out.get_device() == index
                and sx[1] == 1 and sdt[1] == 1 and sb[1] == 1 and sc[1] == 1 and so[1] == 1
                and a.is_contiguous() and state.is_contiguous() and state_out.is_contiguous()):
            for name, v, features in (("x", x, ch), ("dt", dt, ch), ("b", b, narrow), ("c", c, narrow), ("out", out, ch)):
                self._row(name, v, n, features)
            for name, v, want in (("a", a, rates), ("state", state, shape), ("state_out", state_out, shape)):
                self._dense(name, v, want)
        if done is not None:
            self._mask("done", done, (n,))
        self._stream()
        code = self._lib.ssm_scan_step(
            self.h, x.data_ptr(), sx[0], dt.data_ptr(), sdt[0], None if z is None else self._row("z", z, n, ch),
            0 if z is None else z.stride(0), b.data_ptr(), sb[0], c.data_ptr(), sc[0],
            None if done is None else done.data_ptr(), 0 if done is None else done.stride(0), a.data_ptr(),
            None if d is None else self._dense("d", d, (ch,)),
            None if dt_bias is None else self._dense("dt_bias", dt_bias, (ch,)), state.data_ptr(),
            state_out.data_ptr(), out.data_ptr(), so[0], n)
        if code != 0:
            raise SsmError(code, "ssm_scan_step")
        return out
