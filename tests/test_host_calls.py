"""The host side of the C entry points against a stand-in for the CUDA runtime (fake_cudart.c), which
writes down every call with the device that is current: no GPU, and more devices than a machine has.
A library is loaded in a process of its own whose libcudart is the stand-in."""
import ctypes
import os
import subprocess
import sys

import pytest

from paper_2603_12145_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    """Directory with the stand-in as libcudart.so.12; the libraries are built."""
    build.build()
    where = tmp_path_factory.mktemp("fake_cudart")
    (where / "versions").write_text("libcudart.so.12 { global: *; };\n")
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-I" + os.path.join(CUDA, "include"),
                    os.path.join(HERE, "fake_cudart.c"), "-o", str(where / "libcudart.so.12"),
                    "-Wl,-soname,libcudart.so.12", "-Wl,--version-script=" + str(where / "versions")], check=True)
    return str(where)


def child(fake, name):
    """Runs the function of this file in a process that loads the stand-in."""
    env = dict(os.environ, LD_LIBRARY_PATH=fake + os.pathsep + os.environ.get("LD_LIBRARY_PATH", ""), PYTHONPATH=ROOT)
    run = subprocess.run([sys.executable, os.path.abspath(__file__), name, os.path.join(fake, "libcudart.so.12")],
                         cwd=ROOT, env=env, capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stdout + run.stderr


@pytest.mark.parametrize("library", ["ssm", "gated_ffn", "gru_policy", "pong", "cartpole"])
def test_calls_go_to_the_handles_device(fake, library):
    """A handle of device 1, called while device 0 is current, with the default stream (whose value is 0 on
    every device) and with another: everything happens on device 1, and device 0 is current again."""
    child(fake, "device_" + library)


def test_outputs_whose_rows_share_memory_are_refused(fake):
    child(fake, "shared_rows")


def test_long_cases_are_cut_as_they_say(fake):
    """The loops that test_gpu_ssm_long.py is about, by the library's own launches for 148 SMs."""
    child(fake, "cuts")


def test_tiles_of_the_block_are_as_the_cases_say(fake):
    """Of test_gpu_gated_ffn_long.py, with 74 pairs of SMs."""
    child(fake, "tiles")


# ---- in the child: the libraries' own bindings, addresses instead of tensors ---------

class Fake:
    def __init__(self, path):
        self.lib = ctypes.CDLL(path)
        self.lib.fake_what.restype = ctypes.c_char_p
        self.lib.fake_stream.restype = ctypes.c_void_p
        self.lib.fake_stream.argtypes = [ctypes.c_int]

    def current(self):
        v = ctypes.c_int(-1)
        self.lib.cudaGetDevice(ctypes.byref(v))
        return v.value

    def entries(self):
        L = self.lib
        return [(L.fake_what(i).decode(), L.fake_device(i), L.fake_stream(i) or 0, L.fake_blocks(i))
                for i in range(L.fake_count())]

    def on_device_one(self, where, calls, set_stream):
        """calls: (name, function) each; every one has to do something, all of it on device 1."""
        for stream in (None, 0x5000):
            assert set_stream(stream) == 0
            for name, call in calls:
                self.lib.cudaSetDevice(0)
                self.lib.fake_clear()
                code = call()
                assert code == 0, (where, name, code)
                seen = self.entries()
                assert seen, (where, name, "did nothing")
                wrong = [e for e in seen if e[1] != 1]
                assert not wrong, (where, name, "on another device than the handle's", wrong)
                assert all(e[2] == (stream or 0) for e in seen if e[0] == "launch"), (where, name, seen)
                assert self.current() == 0, (where, name, "left another device current")


def address(i):
    return 0x40000000 + 0x1000000 * i


def scan_args(ssm, op, batch, time, channels, states, groups=1):
    """A scan's arguments with every tensor present, [batch][time] order."""
    a = ssm.ScanArgs(batch=batch, time=time)
    wide = lambda i: ssm.Seq(address(i), time * channels, channels)                          # noqa: E731
    narrow = lambda i: ssm.Seq(address(i), time * groups * states, groups * states)          # noqa: E731
    a.x, a.dt, a.z, a.y, a.dy, a.dx, a.ddt, a.dz = [wide(i) for i in range(8)]
    a.b, a.c, a.db, a.dc = [narrow(i) for i in range(8, 12)]
    a.reset = ssm.Seq(address(12), time, 1)
    for i, key in enumerate(("a", "d", "dt_bias", "state", "state_out", "saved", "dstate_out", "da", "dd", "ddt_bias", "dstate")):
        setattr(a, key, address(13 + i))
    a.workspace, a.workspace_bytes = address(30), 1 << 40
    return a


def conv_args(ssm, batch, time, channels):
    a = ssm.ConvArgs(batch=batch, time=time)
    a.x, a.y, a.dy, a.dx = [ssm.Seq(address(i), time * channels, channels) for i in range(4)]
    a.reset = ssm.Seq(address(4), time, 1)
    for i, key in enumerate(("w", "bias", "history", "history_out", "dw", "dbias")):
        setattr(a, key, address(5 + i))
    a.workspace, a.workspace_bytes = address(30), 1 << 40
    return a


def device_ssm(fake):
    from paper_2603_12145_b200 import ssm
    L = ssm.load()
    fake.lib.cudaSetDevice(1)
    h = ssm.ssm_create(96, 16, 1, 4, 1)
    p = address
    for batch, time in ((700, 40), (1, 500)):      # uncut, and cut along the time axis: one kernel, and several
        a, c = scan_args(ssm, h, batch, time, 96, 16), conv_args(ssm, batch, time, 96)
        step = (h, p(0), 96, p(1), 96, p(2), 96, p(3), 16, p(4), 16, p(5), 1, p(6), p(7), p(8), p(9), p(10), p(11), 96, 5)
        fake.on_device_one("ssm", [
            ("scan_forward", lambda: L.ssm_scan_forward(h, ctypes.byref(a))),
            ("scan_backward", lambda: L.ssm_scan_backward(h, ctypes.byref(a))),
            ("scan_step", lambda: L.ssm_scan_step(*step)),
            ("conv_forward", lambda: L.ssm_conv_forward(h, ctypes.byref(c))),
            ("conv_backward", lambda: L.ssm_conv_backward(h, ctypes.byref(c))),
            ("conv_step", lambda: L.ssm_conv_step(h, p(0), 96, p(1), 1, p(2), p(3), p(4), p(5), p(6), 96, 5)),
        ], lambda s: L.ssm_set_stream(h, s))


def shared_rows(fake):
    """Strides of outputs [batch][time][features]: rows of one order, of the other and of wider arrays are
    taken; two rows at the same place, or running into each other, are not (they would be written in no order)."""
    from paper_2603_12145_b200 import ssm
    L = ssm.load()
    ch, states, batch, time = 96, 16, 3, 5
    h = ssm.ssm_create(ch, states, 1, 4, 1)

    def strides(row):
        good = [(time * row, row), (row, batch * row), (time * (row + 5), row + 5), (row + 7, batch * (row + 7)),
                (7 * time * row, row), (row, 9 * batch * row), ((time - 1) * row + row, row)]
        bad = [(row, row), (0, row), (row, 0), (2 * row, row), (row, 2 * row), (time * row - 1, row), (row, batch * row - 1),
               (row - 1, batch * row), (time * row, row - 1), (4 * row, row), (row, 2 * row + 1)]
        return good, bad

    scan = {"y": (L.ssm_scan_forward, ch), "dx": (L.ssm_scan_backward, ch), "ddt": (L.ssm_scan_backward, ch),
            "dz": (L.ssm_scan_backward, ch), "db": (L.ssm_scan_backward, states), "dc": (L.ssm_scan_backward, states)}
    conv = {"y": (L.ssm_conv_forward, ch), "dx": (L.ssm_conv_backward, ch)}
    for kind, outputs in (("scan", scan), ("conv", conv)):
        for key, (call, row) in outputs.items():
            good, bad = strides(row)
            for taken, pairs in ((0, good), (-1, bad)):
                for pair in pairs:
                    a = scan_args(ssm, h, batch, time, ch, states) if kind == "scan" else conv_args(ssm, batch, time, ch)
                    setattr(a, key, ssm.Seq(address(40), *pair))
                    assert call(h, ctypes.byref(a)) == taken, (kind, key, row, pair)
    # neither order's rows lie together, and none share memory: 0, 2, 4 and 3, 5, 7; with a fourth step 6 would meet 3 + 3
    for b, t, taken in ((2, 3, 0), (3, 4, -1), (3, 2, 0)):
        a = conv_args(ssm, b, t, ch)
        a.y = ssm.Seq(address(40), 3 * ch, 2 * ch)
        assert L.ssm_conv_forward(h, ctypes.byref(a)) == taken, (b, t)
    # of a single row or step the strides do not matter
    for b, t, pair in ((1, 5, (0, ch)), (3, 1, (ch, 0)), (1, 1, (0, 0))):
        a = conv_args(ssm, b, t, ch)
        a.y = ssm.Seq(address(40), *pair)
        assert L.ssm_conv_forward(h, ctypes.byref(a)) == 0, (b, t, pair)


def up(a, b):
    return -(-a // b)


def cuts(fake):
    import test_gpu_ssm_long as cases
    from paper_2603_12145_b200 import ssm
    L = ssm.load()
    for batch, time, ch, n, groups, _, _, forward, backward in cases.SCAN:
        h = ssm.ssm_create(ch, n, groups, 4, 0)
        lanes, quads = (1 if n <= 16 else 2 if n <= 32 else 4), next(q for q in (1, 2, 4, 8, 16) if 4 * q >= n)
        chunks = up(time, 16)
        assert up(chunks, forward[1]) == forward[0] and up(chunks, backward[1]) == backward[0]
        a = scan_args(ssm, h, batch, time, ch, n, groups)
        fake.lib.fake_clear()
        assert L.ssm_scan_forward(h, ctypes.byref(a)) == 0
        blocks = batch * forward[0] * groups * up(ch // groups, 128 // lanes)
        assert [e[3] for e in fake.entries() if e[0] == "launch"][-1] == blocks, (batch, time, fake.entries())
        fake.lib.fake_clear()
        assert L.ssm_scan_backward(h, ctypes.byref(a)) == 0
        blocks = backward[2] * groups * up(ch // groups, 96 if 16 < n <= 32 else 128)
        launches = [e[3] for e in fake.entries() if e[0] == "launch"]
        assert len(launches) == (3 if backward[0] == 1 else 5) and launches[-3] == blocks, (batch, time, launches, blocks)
        carry = batch * backward[0] * ch * (16 * quads + 4) if backward[0] > 1 else 0
        total = L.ssm_scan_workspace_bytes(h, batch, time, 1)
        parts = up(ch // groups, 96 if 16 < n <= 32 else 128) * batch * time * groups * 2 * max(16, 4 * quads) * 4
        assert abs(total - carry - backward[2] * ch * (16 * quads + 8) - parts) < 64, (batch, time, total)
    assert any(c[8][2] < c[0] * c[8][0] for c in cases.SCAN) and any(c[7][0] > 1 and c[7][1] > 1 for c in cases.SCAN)
    p = address
    for n, ch, states, groups, _, rows in cases.STEPS:
        h = ssm.ssm_create(ch, states, groups, 4, 0)
        fake.lib.fake_clear()
        assert L.ssm_scan_step(h, p(0), ch, p(1), ch, p(2), ch, p(3), groups * states, p(4), groups * states, p(5), 1, p(6), p(7),
                               p(8), p(9), p(10), p(11), ch, n) == 0
        lanes = next(q for q in (1, 2, 4, 8, 16) if 4 * q >= states)
        assert [e[3] for e in fake.entries()] == [up(ch, 256 // lanes) * up(n, rows)], (n, ch, fake.entries(), rows)
    assert any(c[5] > 4 for c in cases.STEPS)
    for batch, time, ch, width, _, _, run, runs in cases.CONV:
        h = ssm.ssm_create(ch, 16, 1, width, 0)
        c = conv_args(ssm, batch, time, ch)
        fake.lib.fake_clear()
        assert L.ssm_conv_forward(h, ctypes.byref(c)) == 0
        warps = up(ch // 4, 32) if ch % 4 == 0 else up(ch, 32)
        units = batch * up(time, run)
        assert [e[3] for e in fake.entries()] == [up(units * warps, 4)], (batch, time, fake.entries())
        slots = L.ssm_conv_workspace_bytes(h, batch, time) // (4 * ch * (width + 1))
        assert up(units, slots) == runs, (batch, time, units, slots)
    assert any(c[6] > 8 for c in cases.CONV) and all(c[7] > 1 for c in cases.CONV)


def device_gated_ffn(fake):
    from paper_2603_12145_b200 import gated_ffn
    L = gated_ffn.load()
    p = address
    for type_ in (0, 1):
        fake.lib.cudaSetDevice(1)
        h = gated_ffn.gated_ffn_create(200, 136, type_, type_)
        calls = []
        for n in (5, 300):                          # the streaming kernel, and the tiles
            calls += [("forward %d" % n, lambda n=n: L.gated_ffn_forward(h, p(0), 200, p(1), p(2), p(3), p(4), p(5), 200, p(6),
                                                                         1 << 30, n)),
                      ("backward %d" % n, lambda n=n: L.gated_ffn_backward(h, p(7), 200, p(0), 200, p(1), p(2), p(3), p(4), p(5),
                                                                           200, p(8), p(9), p(6), 1 << 30, n))]
        fake.on_device_one("gated_ffn", calls + [("status", lambda: L.gated_ffn_status(h))],
                           lambda s: L.gated_ffn_set_stream(h, s))
        fake.lib.fake_clear()
        assert L.gated_ffn_destroy(h) == 0
        assert fake.entries() and all(e[1] == 1 for e in fake.entries()) and fake.current() == 0, fake.entries()


def host(np, *shape):
    v = np.zeros(shape, dtype=np.float32)
    return v, v.ctypes.data


def device_gru_policy(fake):
    import numpy as np
    from paper_2603_12145_b200 import gru_policy
    L = gru_policy.load()
    shapes = {"enc_w": (64, 6), "enc_b": (64,), "w_ih": (192, 64), "w_hh": (192, 64), "b_ih": (192,), "b_hh": (192,),
              "head_w": (3, 64), "head_b": (3,)}
    fake.lib.cudaSetDevice(1)
    h = gru_policy.gru_policy_create(64, 6, 3, {k: np.zeros(v, dtype=np.float32) for k, v in shapes.items()})
    p = address
    fake.on_device_one("gru_policy", [
        ("encode", lambda: L.gru_policy_encode(h, p(0), p(1), p(2), p(3), 300)),
        ("cell", lambda: L.gru_policy_cell(h, p(0), p(1), p(2), 300)),
        ("cell_head", lambda: L.gru_policy_cell_head(h, p(0), p(1), p(2), p(3), p(4), 300)),
        ("head", lambda: L.gru_policy_head(h, p(0), p(1), 300)),
        ("status", lambda: L.gru_policy_status(h)),
    ], lambda s: L.gru_policy_set_stream(h, s))
    fake.lib.fake_clear()
    assert L.gru_policy_destroy(h) == 0
    assert fake.entries() and all(e[1] == 1 for e in fake.entries()) and fake.current() == 0, fake.entries()


def device_pong(fake):
    import numpy as np
    from paper_2603_12145_b200 import pong
    L = pong.load()
    p, n = address, 200
    for pixels in (0, 1):
        h = ctypes.c_void_p()
        fake.lib.cudaSetDevice(1)
        assert L.pong_create_ex(ctypes.byref(h), n, 7, ctypes.byref(pong._Config(pixels, 1, 0))) == 0
        keep, obs = host(np, n * 4 * 84 * 84 + 8 * n * 6)
        rest, reward = host(np, 8 * n)
        state, got = np.zeros((11, n), dtype=np.int32), np.zeros((11, n), dtype=np.int32)
        state[2] = 512                               # the ball's speed at a serve
        fake.on_device_one("pong", [
            ("reset", lambda: L.pong_reset(h, p(0))),
            ("step", lambda: L.pong_step(h, p(3), p(0), p(1), p(2))),
            ("rollout", lambda: L.pong_rollout(h, 8, 0, None, p(0), p(1), p(2))),
            ("rollout_host", lambda: L.pong_rollout_host(h, 8, 0, None, obs, reward, reward)),
            ("fill_actions", lambda: L.pong_fill_actions(h, 8, 0, p(0))),
            ("fill_words", lambda: L.pong_fill_words(h, 8, p(0))),
            ("sample_actions", lambda: L.pong_sample_actions(h, p(0), p(1), p(2))),
            ("episode_stats", lambda: L.pong_episode_stats(h, None, None, None, 1)),
            ("get_state", lambda: L.pong_get_state(h, got.ctypes.data, None)),
            ("set_state", lambda: L.pong_set_state(h, state.ctypes.data, 0)),
        ], lambda s: L.pong_set_stream(h, s))
        fake.lib.fake_clear()
        assert L.pong_destroy(h) == 0
        assert fake.entries() and all(e[1] == 1 for e in fake.entries()) and fake.current() == 0, fake.entries()
        del keep, rest


def device_cartpole(fake):
    import numpy as np
    from paper_2603_12145_b200 import cartpole
    L = cartpole.load()
    p = address
    for n in (200, 65536):                           # blocks, and the balanced chains with their own limit
        h = ctypes.c_void_p()
        fake.lib.cudaSetDevice(1)
        assert L.cartpole_create(ctypes.byref(h), n, 7, 0) == 0
        keep, obs = host(np, 8 * n * 4)
        rest, reward = host(np, 8 * n)
        f, i = np.zeros((4, n), dtype=np.float32), np.zeros((2, n), dtype=np.int32)
        fake.on_device_one("cartpole", [
            ("reset", lambda: L.cartpole_reset(h, p(0))),
            ("step", lambda: L.cartpole_step(h, p(3), p(0), p(1), p(2))),
            ("rollout", lambda: L.cartpole_rollout(h, 8, 0, None, p(0), p(1), p(2))),
            ("rollout_host", lambda: L.cartpole_rollout_host(h, 8, 0, None, obs, reward, reward)),
            ("episode_stats", lambda: L.cartpole_episode_stats(h, None, None, 1)),
            ("get_state", lambda: L.cartpole_get_state(h, f.ctypes.data, i.ctypes.data, None)),
            ("set_state", lambda: L.cartpole_set_state(h, f.ctypes.data, i.ctypes.data, 0)),
        ], lambda s: L.cartpole_set_stream(h, s))
        fake.lib.fake_clear()
        assert L.cartpole_destroy(h) == 0
        assert fake.entries() and all(e[1] == 1 for e in fake.entries()) and fake.current() == 0, fake.entries()
        del keep, rest


def tiles(fake):
    import test_gpu_gated_ffn_long as cases
    from paper_2603_12145_b200 import gated_ffn
    L = gated_ffn.load()
    p = address
    for n, model, hidden, activation, _, forward, slope in cases.TILES:
        h = gated_ffn.gated_ffn_create(model, hidden, 0, 0)
        fake.lib.fake_clear()
        assert L.gated_ffn_forward(h, p(0), model, p(1), p(2), p(3), p(4), p(5), model, p(6), 1 << 40, n) == 0
        grid = fake.entries()[0][3]
        count = up(n, 256) * up(hidden, 128)
        assert (grid // 2, up(count, grid // 2)) == forward, (n, hidden, grid, count)
        fake.lib.fake_clear()
        assert L.gated_ffn_backward(h, p(0), model, p(1), model, p(2), p(3), p(4), p(5), p(6), model, p(7), p(8), p(9), 1 << 40, n) == 0
        grid = fake.entries()[0][3]
        count = up(n, 256) * up(hidden, 192)
        assert (grid // 2, up(count, grid // 2)) == slope, (n, hidden, grid, count)
    assert any(c[5][1] > 1 for c in cases.TILES) and any(c[6][1] > 1 for c in cases.TILES)


if __name__ == "__main__":
    globals()[sys.argv[1]](Fake(sys.argv[2]))
