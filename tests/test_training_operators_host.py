"""The training operators without a GPU: the libraries' symbols, the argument checks that come before any CUDA call, the
host side against a stand-in for the CUDA runtime (see test_host_calls.py; a process with torch has the real one)."""
import ctypes
import os
import subprocess
import sys

import pytest

from paper_2603_12145_b200 import build, gated_recurrence, layer_norm, orthogonal
from test_abi import declared_symbols
from test_host_calls import Fake, address, fake  # noqa: F401

LIBRARIES = {"layer_norm": layer_norm, "gated_recurrence": gated_recurrence, "orthogonal": orthogonal}
ERRORS = {"layer_norm": layer_norm.LayerNormError, "gated_recurrence": gated_recurrence.GatedRecurrenceError,
          "orthogonal": orthogonal.OrthogonalError}


@pytest.mark.parametrize("name", LIBRARIES)
def test_library_exports_every_declared_symbol(name):
    lib = ctypes.CDLL(build.build_one("lib%s_b200.so" % name))
    names = declared_symbols(name + ".h", name)
    assert len(names) >= 8 and set(names) == set(LIBRARIES[name].EXPORTS)
    for symbol in names:
        assert hasattr(lib, symbol), symbol
    module = LIBRARIES[name]
    module.load(build_if_missing=True)
    assert module.strerror(0) == "ok" and module.strerror(-99) == "unknown error"
    assert all(module.strerror(code) != "unknown error" for code in range(-5, 0))


def test_checks_before_any_cuda_call():
    h = ctypes.c_void_p()
    L = layer_norm.load(build_if_missing=True)
    assert L.layer_norm_create(None, 64, 1e-5, 0) == -2
    for width, eps, kind in ((0, 1e-5, 0), (8193, 1e-5, 0), (64, 0.0, 0), (64, float("nan"), 0), (64, float("inf"), 0), (64, 1e-5, 3)):
        assert L.layer_norm_create(ctypes.byref(h), width, eps, kind) == -1
    assert L.layer_norm_destroy(None) == -2 and L.layer_norm_set_stream(None, None) == -2
    assert L.layer_norm_workspace_bytes(None, 1) == 0 and L.layer_norm_launch_count(None) == 0
    L = gated_recurrence.load(build_if_missing=True)
    assert L.gated_recurrence_create(None, 64, 0) == -2
    for channels, kind in ((0, 0), (65537, 0), (64, 3), (64, -1)):
        assert L.gated_recurrence_create(ctypes.byref(h), channels, kind) == -1
    assert L.gated_recurrence_forward(None, None) == -2 and L.gated_recurrence_destroy(None) == -2
    assert L.gated_recurrence_saved_bytes(None, 1, 1) == 0
    L = orthogonal.load(build_if_missing=True)
    usual = (3.4445, -4.775, 2.0315, 1e-7, 0)
    assert L.orthogonal_create(None, 4, 4, 5, *usual) == -2
    for bad in ((0, 4, 5) + usual, (4, 65537, 5) + usual, (4, 4, 0) + usual, (4, 4, 33) + usual, (4, 4, 5) + usual[:3] + (0.0, 0),
                (4, 4, 5) + usual[:4] + (3,), (4, 4, 5, float("inf")) + usual[1:]):
        assert L.orthogonal_create(ctypes.byref(h), *bad) == -1
    assert L.orthogonal_destroy(None) == -2 and L.orthogonal_status(None) == -2
    assert L.orthogonal_workspace_bytes(None, 1) == 0


def test_no_cpu_fallback():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is present")
    for name, module in LIBRARIES.items():
        module.load(build_if_missing=True)
        args = {"layer_norm": (64, 1e-5, 0), "gated_recurrence": (64, 0), "orthogonal": (64, 64, 5, 3.4445, -4.775, 2.0315, 1e-7, 0)}[name]
        with pytest.raises(ERRORS[name]) as ei:
            getattr(module, name + "_create")(*args)
        assert ei.value.code == -4
    for make in (lambda: layer_norm.LayerNorm(64, device="cpu"), lambda: gated_recurrence.GatedRecurrence(64, device="cpu"),
                 lambda: orthogonal.Orthogonal(64, 64, device="cpu")):
        with pytest.raises(ValueError):
            make()


# ---- against the stand-in for the CUDA runtime ----------------------------------------

def child(fake, name):                                                                   # noqa: F811
    env = dict(os.environ, LD_LIBRARY_PATH=fake + os.pathsep + os.environ.get("LD_LIBRARY_PATH", ""),
               PYTHONPATH=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    run = subprocess.run([sys.executable, os.path.abspath(__file__), name, os.path.join(fake, "libcudart.so.12")],
                         env=env, capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stdout + run.stderr


@pytest.mark.parametrize("name", ["device_calls", "argument_checks", "shared_rows", "cuts"])
def test_host_side(fake, name):                                                          # noqa: F811
    child(fake, name)


def recurrence_args(batch, time, ch):
    a = gated_recurrence.Args(batch=batch, time=time)
    for i, key in enumerate(("x", "r", "i", "y", "dy", "dx", "dr", "di")):
        setattr(a, key, gated_recurrence.Seq(address(i), time * ch, ch))
    a.reset = gated_recurrence.Seq(address(8), time, 1)
    for i, key in enumerate(("a", "state", "state_out", "saved", "dstate_out", "da", "dstate")):
        setattr(a, key, address(9 + i))
    a.workspace, a.workspace_bytes = address(20), 1 << 40
    return a


def device_calls(fake):                                                                  # noqa: F811
    p = address
    L = layer_norm.load()
    for kind, width in ((0, 100), (1, 576), (2, 4096)):
        fake.lib.cudaSetDevice(1)
        h = layer_norm.layer_norm_create(width, 1e-5, kind)
        fake.on_device_one("layer_norm", [
            ("forward", lambda: L.layer_norm_forward(h, p(0), width, p(1), width, p(2), p(3), p(4), width, p(5), width, p(6), 300)),
            ("backward", lambda: L.layer_norm_backward(h, p(0), width, p(1), width, p(2), p(6), p(3), width, p(4), width, p(7),
                                                       p(8), p(9), 1 << 40, 300)),
        ], lambda s: L.layer_norm_set_stream(h, s))
    L = gated_recurrence.load()
    for kind in (0, 1, 2):
        fake.lib.cudaSetDevice(1)
        h = gated_recurrence.gated_recurrence_create(96, kind)
        for batch, time in ((700, 40), (1, 500)):
            a = recurrence_args(batch, time, 96)
            fake.on_device_one("gated_recurrence", [
                ("forward", lambda: L.gated_recurrence_forward(h, ctypes.byref(a))),
                ("backward", lambda: L.gated_recurrence_backward(h, ctypes.byref(a))),
                ("step", lambda: L.gated_recurrence_step(h, p(0), 96, p(1), 96, p(2), 96, p(3), 1, p(4), p(5), p(6), p(7), 96, 5)),
            ], lambda s: L.gated_recurrence_set_stream(h, s))
    L = orthogonal.load()
    for rows, cols, batch in ((64, 384, 3), (1728, 576, 1), (2048, 1000, 1), (20, 5000, 2)):
        fake.lib.cudaSetDevice(1)
        h = orthogonal.orthogonal_create(rows, cols, 5, 3.4445, -4.775, 2.0315, 1e-7, 1)
        size = L.orthogonal_workspace_bytes(h, batch)
        fake.on_device_one("orthogonal", [
            ("update", lambda: L.orthogonal_update(h, p(0), rows * cols, cols, p(10), rows * cols, cols, p(20), size, batch)),
            ("status", lambda: L.orthogonal_status(h)),
        ], lambda s: L.orthogonal_set_stream(h, s))
        fake.lib.fake_clear()
        assert L.orthogonal_destroy(h) == 0
        assert fake.entries() and all(e[1] == 1 for e in fake.entries()) and fake.current() == 0, fake.entries()


def argument_checks(fake):                                                               # noqa: F811
    """Pointers, alignments, strides and workspaces: refused before anything is launched."""
    p = address
    L = layer_norm.load()
    h = layer_norm.layer_norm_create(100, 1e-5, 1)

    def forward(x=p(0), sx=100, r=p(1), sr=100, w=p(2), b=p(3), t=p(4), st=100, y=p(5), sy=100, kept=p(6), n=30):
        return L.layer_norm_forward(h, x, sx, r, sr, w, b, t, st, y, sy, kept, n)

    def backward(dy=p(0), sdy=100, s=p(1), ss=100, w=p(2), kept=p(3), d=p(4), sd=100, dx=p(5), sdx=100, dw=p(6), db=p(7), ws=p(8),
                 size=1 << 30, n=30):
        return L.layer_norm_backward(h, dy, sdy, s, ss, w, kept, d, sd, dx, sdx, dw, db, ws, size, n)

    def refused(call, cases):
        for code, kw in cases:
            fake.lib.fake_clear()
            assert call(**kw) == code, (call.__name__, kw)
            assert not [e for e in fake.entries() if e[0] == "launch"], kw

    assert forward() == 0 and forward(r=None, t=None) == 0 and forward(w=None, b=None, kept=None) == 0 and forward(n=1, sy=0, st=0) == 0
    refused(forward, [(-1, dict(n=0)), (-1, dict(n=1 << 31)), (-2, dict(x=None)), (-2, dict(y=None)), (-2, dict(r=None)), (-2, dict(t=None)),
                      (-1, dict(sx=-1)), (-1, dict(sy=99)), (-1, dict(st=50)), (-3, dict(x=p(0) + 1)), (-3, dict(w=p(2) + 2)),
                      (-3, dict(kept=p(6) + 4)), (-3, dict(t=p(4) + 1))])
    assert backward() == 0 and backward(d=None) == 0 and backward(dw=None, db=None, ws=None, size=0) == 0
    need = L.layer_norm_workspace_bytes(h, 30)
    assert backward(size=need) == 0
    refused(backward, [(-1, dict(n=0)), (-2, dict(dy=None)), (-2, dict(s=None)), (-2, dict(kept=None)), (-2, dict(dx=None)), (-2, dict(dw=None)),
                       (-2, dict(ws=None)), (-5, dict(size=need - 1)), (-1, dict(sdx=99)), (-1, dict(sd=-1)), (-3, dict(ws=p(8) + 8)),
                       (-3, dict(kept=p(3) + 4))])
    L = gated_recurrence.load()
    h = gated_recurrence.gated_recurrence_create(96, 1)
    for call in (L.gated_recurrence_forward, L.gated_recurrence_backward):
        assert call(h, ctypes.byref(recurrence_args(3, 500, 96))) == 0
        for code, key, value in ((-1, "batch", 0), (-1, "time", 0), (-1, "time", 1 << 31), (-2, "a", None), (-3, "a", p(9) + 2),
                                 (-3, "workspace", p(20) + 8), (-2, "workspace", None), (-5, "workspace_bytes", 8),
                                 (-2, "x", gated_recurrence.Seq(None, 1, 1)), (-1, "r", gated_recurrence.Seq(p(1), -1, 96)),
                                 (-3, "i", gated_recurrence.Seq(p(2) + 1, 48000, 96))):
            a = recurrence_args(3, 500, 96)
            setattr(a, key, value)
            fake.lib.fake_clear()
            assert call(h, ctypes.byref(a)) == code, (key, value)
            assert not [e for e in fake.entries() if e[0] == "launch"], key
    a = recurrence_args(3, 500, 96)
    a.state_out = a.state
    assert L.gated_recurrence_forward(h, ctypes.byref(a)) == -1
    for key in ("saved", "da"):
        a = recurrence_args(3, 500, 96)
        setattr(a, key, None)
        assert L.gated_recurrence_backward(h, ctypes.byref(a)) == -2
    L = orthogonal.load()
    small = orthogonal.orthogonal_create(50, 160, 5, 3.4445, -4.775, 2.0315, 1e-7, 1)      # stays on the chip: no workspace
    assert L.orthogonal_workspace_bytes(small, 2) == 0
    assert L.orthogonal_update(small, p(0), 8000, 160, p(1), 8000, 160, None, 0, 2) == 0
    h = orthogonal.orthogonal_create(150, 160, 5, 3.4445, -4.775, 2.0315, 1e-7, 1)
    need = L.orthogonal_workspace_bytes(h, 2)

    def update(g=p(0), gb=24000, gr=160, o=p(1), ob=24000, orow=160, ws=p(2), size=need, n=2):
        return L.orthogonal_update(h, g, gb, gr, o, ob, orow, ws, size, n)

    assert update() == 0 and update(gb=0) == 0 and update(n=1, ob=0) == 0
    refused(update, [(-1, dict(n=0)), (-1, dict(n=65536)), (-2, dict(g=None)), (-2, dict(o=None)), (-2, dict(ws=None)), (-1, dict(gr=-1)),
                     (-1, dict(orow=159)), (-1, dict(ob=23999)), (-3, dict(g=p(0) + 1)), (-3, dict(ws=p(2) + 128)), (-5, dict(size=need - 1))])


def shared_rows(fake):                                                                   # noqa: F811
    L = gated_recurrence.load()
    ch, batch, time = 96, 3, 5
    h = gated_recurrence.gated_recurrence_create(ch, 1)
    good = [(time * ch, ch), (ch, batch * ch), (time * (ch + 5), ch + 5), ((time - 1) * ch + ch, ch)]
    bad = [(ch, ch), (0, ch), (ch, 0), (2 * ch, ch), (time * ch - 1, ch), (ch - 1, batch * ch)]
    for key, call in (("y", L.gated_recurrence_forward), ("dx", L.gated_recurrence_backward), ("dr", L.gated_recurrence_backward),
                      ("di", L.gated_recurrence_backward)):
        for taken, pairs in ((0, good), (-1, bad)):
            for pair in pairs:
                a = recurrence_args(batch, time, ch)
                setattr(a, key, gated_recurrence.Seq(address(40), *pair))
                assert call(h, ctypes.byref(a)) == taken, (key, pair)


def cuts(fake):                                                                          # noqa: F811
    """A call that is cut along the time axis takes two more kernels, one with rows enough does not; workspaces fit."""
    L = gated_recurrence.load()
    h = gated_recurrence.gated_recurrence_create(96, 1)
    for batch, time, forward, backward in ((5000, 40, 1, 2), (1, 500, 3, 4), (1, 1, 1, 2), (2, 31, 1, 2), (3, 777, 3, 4)):
        a = recurrence_args(batch, time, 96)
        for call, want in ((L.gated_recurrence_forward, forward), (L.gated_recurrence_backward, backward)):
            fake.lib.fake_clear()
            assert call(h, ctypes.byref(a)) == 0
            assert len([e for e in fake.entries() if e[0] == "launch"]) == want, (batch, time, fake.entries())
        assert L.gated_recurrence_saved_bytes(h, batch, time) == batch * -(-time // 4) * 96 * 4


if __name__ == "__main__":
    globals()[sys.argv[1]](Fake(sys.argv[2]))
