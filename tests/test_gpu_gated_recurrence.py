"""The gated linear recurrence against the binary64 oracle, through the binding.

Tolerances.  u = 2^-24; u_T is the type's half step (2^-8, 2^-11, 2^-24).  A sigmoid has at most 8 u of relative error (two
of the exponential, one of 1 + e, two of the reciprocal, the products; |argument| u more where the argument is of 16 bits),
L one more, e^L - 1 at most 8 u beyond L's (the large branch doubles the exponential's error), the gain half of that and its
square root's 5, the input term both gates': C = 64 covers every factor with arguments up to 8.  An error of e^L - 1 enters
as (C |e^L - 1| + 2) u of the state, that of e^L itself is absolute: C (e^L + 0.3) u.  Carried along the recurrences of the
magnitudes (every term by its absolute value), H of the states and G of their gradients:

    D_t = e^L D_{t-1} + (C |e^L - 1| + 2) H_{t-1} + C v_t             for h, in units of u; likewise for g
    dx, di: (D_g + C G) times their factors
    dL: D_g e^L (H + w) + G [e^L D + C (e^L + 0.3)(H + w)],   w = |u_t| e^L / k_t;    dr: that and C once more
    da: the sum of dL's, and R u sum |dL sigmoid(r)| with R = 64 + steps / 8 roundings of the sum (eight steps are
        summed by themselves, and a warp's pieces then one after the other)
"""
import numpy as np
import pytest

from oracle import training as tr
from paper_2603_12145_b200 import gated_recurrence

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
UNIT = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
C = 64.0


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    gated_recurrence.load(build_if_missing=True)
    return torch


def f64(t):
    return t.double().cpu().numpy()


def rounded(torch, a, dtype, layout="batch"):
    """(device tensor of the type, its values).  layout: "batch", "time" (a transposed [time, batch, channels]) or
    "wide" (columns of a wider array, at an odd offset)."""
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda().to(getattr(torch, dtype))
    values = f64(t)
    if layout == "time":
        t = t.transpose(0, 1).contiguous().transpose(0, 1)
    elif layout == "wide":
        wide = torch.full(t.shape[:-1] + (t.shape[-1] + 5,), float("nan"), dtype=t.dtype, device=t.device)
        wide[..., 3:3 + t.shape[-1]] = t
        t = wide[..., 3:3 + t.shape[-1]]
    return t, values


def make(torch, seed, batch, time, ch, dtype, layout="batch", reset=0.0, carry=False):
    r = np.random.Generator(np.random.PCG64(seed))
    dev, val = {}, {}
    for name, shift in (("x", 0.0), ("r", 0.5), ("i", 0.0), ("dy", 0.0)):
        dev[name], val[name] = rounded(torch, np.clip(r.standard_normal((batch, time, ch)) * 1.5 + shift, -7, 7), dtype, layout)
    params = {"a": -np.exp(r.uniform(np.log(1e-4), np.log(8.0), ch)), "state": r.standard_normal((batch, ch)),
              "dstate_out": r.standard_normal((batch, ch))}
    for name, v in params.items():
        dev[name], val[name] = rounded(torch, v, "float32")
    if not carry:
        for name in ("state", "dstate_out"):
            dev[name] = val[name] = None
    dev["reset"] = val["reset"] = None
    if reset:
        m = (r.random((batch, time)) < reset).astype(np.uint8)
        val["reset"] = m
        t = torch.from_numpy(m).cuda()
        dev["reset"] = t.t().contiguous().t() if layout == "time" else t
    return dev, val


def bounds(v):
    """Error bounds in units of u for y, state, and the gradients (da without the rounding of its sum) and the
    magnitude of da's terms."""
    x, batch, time = np.abs(v["x"]), v["x"].shape[0], v["x"].shape[1]
    fresh = np.zeros((batch, time, 1), bool) if v["reset"] is None else v["reset"][:, :, None] != 0
    sr, si = tr.sigmoid(v["r"]), tr.sigmoid(v["i"])
    L = v["a"] * sr
    al, e = np.exp(L), -np.expm1(L)
    k = np.sqrt(-np.expm1(2 * L))
    term = k * si * x
    zero = np.zeros_like(x[:, 0])
    h, d = (zero if v["state"] is None else np.abs(v["state"])), zero
    before, dbefore, out = np.empty_like(x), np.empty_like(x), {"y": np.empty_like(x)}
    for t in range(time):
        h, d = np.where(fresh[:, t], 0.0, h), np.where(fresh[:, t], 0.0, d)
        before[:, t], dbefore[:, t] = h, d
        d = al[:, t] * d + (C * e[:, t] + 2) * h + C * term[:, t]
        h = al[:, t] * h + term[:, t]
        out["y"][:, t] = d
    out["state"] = d
    for key in ("dx", "dr", "di"):
        out[key] = np.empty_like(x)
    out["da"], sums = np.zeros(x.shape[2]), np.zeros(x.shape[2])
    g, dg = (zero if v["dstate_out"] is None else np.abs(v["dstate_out"])), zero
    for t in range(time - 1, -1, -1):
        g, dg = g + np.abs(v["dy"][:, t]), dg + g + np.abs(v["dy"][:, t])      # one rounding of the sum
        a, s, xx = al[:, t], si[:, t], x[:, t]
        out["dx"][:, t] = (dg + C * g) * k[:, t] * s
        out["di"][:, t] = (dg + C * g) * k[:, t] * s * xx * (1 - s)
        w = s * xx * a / np.maximum(k[:, t], 1e-30)
        dl = dg * a * (before[:, t] + w) + g * (a * dbefore[:, t] + C * (a + 0.3) * (before[:, t] + w))
        m = g * a * (before[:, t] + w)
        out["dr"][:, t] = (dl + C * m) * np.abs(L[:, t]) * (1 - sr[:, t])
        out["da"] += (dl * sr[:, t]).sum(axis=0)
        sums += (m * sr[:, t]).sum(axis=0)
        dg = a * dg + (C * e[:, t] + 2) * g
        g = a * g
        g, dg = np.where(fresh[:, t], 0.0, g), np.where(fresh[:, t], 0.0, dg)
    out["dstate"] = dg
    return out, sums


def near(name, got, want, units, dtype="float32"):
    got = f64(got)
    tol = UNIT[dtype] * np.abs(want) * 1.01 + U * units + (2.0 ** -25 if dtype == "float16" else 1e-37)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, first at %s: got %r want %r tol %r" % (
        name, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0],
        np.broadcast_to(tol, got.shape)[bad][0])


def check_all(torch, op, dev, val, dtype):
    batch, time, ch = dev["x"].shape
    four = [dev[k] for k in ("x", "r", "i", "a")]
    v4 = [val[k] for k in ("x", "r", "i", "a")]
    saved, last = op.saved(batch, time), op.state(batch)
    y = op.sequence(*four, reset=dev["reset"], state=dev["state"], state_out=last, saved=saved)
    g = op.backward(dev["dy"], *four, saved, reset=dev["reset"], dstate_out=dev["dstate_out"],
                    want_dstate=dev["state"] is not None)
    torch.cuda.synchronize()
    units, sums = bounds(val)
    want_y, want_last, _ = tr.recurrence(*v4, val["reset"], val["state"])
    near("y", y, want_y, units["y"], dtype)
    near("state", last, want_last, units["state"])
    want = tr.recurrence_grad(val["dy"], *v4, val["reset"], val["state"], val["dstate_out"])
    for key in ("dx", "dr", "di"):
        near(key, g[key], want[key], units[key], dtype)
    near("da", g["da"], want["da"], units["da"] + (64 + batch * time / 8) * sums)
    if dev["state"] is not None:
        near("dstate", g["dstate"], want["dstate"], units["dstate"])
    else:
        assert g["dstate"] is None
    return y, last, g


CASES = [
    # batch, time, channels, dtype, layout, reset, carry
    (1, 1, 1, "float32", "batch", 0, False),
    (2, 1, 40, "bfloat16", "time", 0, True),
    (1, 7, 130, "float32", "batch", 0, True),
    (3, 8, 64, "bfloat16", "batch", 0.2, True),
    (3, 9, 66, "float16", "time", 0.1, True),
    (2, 65, 96, "float16", "wide", 0.05, True),
    (2, 70, 35, "float32", "wide", 0.1, False),
    (5, 40, 129, "bfloat16", "time", 0.1, True),
    (2, 33, 20, "bfloat16", "batch", 1.0, True),      # every step starts an episode
    (1, 600, 33, "float32", "batch", 0.004, True),    # one row: the time axis is cut
    (1, 1000, 64, "bfloat16", "batch", 0, False),
    (3, 333, 50, "float16", "time", 0.01, True),
    (300, 40, 257, "bfloat16", "time", 0.05, True),
    (2500, 19, 70, "float32", "batch", 0.05, True),   # several rows per warp backward
    (400, 11, 576, "bfloat16", "time", 0.02, False),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_sequence_and_gradients(torch, case):
    batch, time, ch, dtype, layout, reset, carry = case
    dev, val = make(torch, 10 + time, batch, time, ch, dtype, layout, reset, carry)
    op = gated_recurrence.GatedRecurrence(ch, dtype=getattr(torch, dtype))
    y, last, g = check_all(torch, op, dev, val, dtype)
    again = check_all(torch, op, dev, val, dtype)
    assert torch.equal(again[0], y) and torch.equal(again[1], last)
    assert all(torch.equal(again[2][k], g[k]) for k in g if g[k] is not None)


@pytest.mark.parametrize("case", [(1, 16000, 64, "bfloat16", "batch", 0, True), (1, 16000, 40, "float32", "batch", 0.0005, True),
                                  (2, 9000, 70, "float16", "time", 0.001, True), (1, 9000, 300, "bfloat16", "wide", 0, False)], ids=str)
def test_many_segments(torch, case):
    """Long rows in few channels, cut into so many segments that runs of them are chained, with and without resets."""
    batch, time, ch, dtype, layout, reset, carry = case
    dev, val = make(torch, 10 + time, batch, time, ch, dtype, layout, reset, carry)
    check_all(torch, gated_recurrence.GatedRecurrence(ch, dtype=getattr(torch, dtype)), dev, val, dtype)


def test_single_tokens_are_the_sequence(torch):
    """Step by step from the same state, in place, with the flags of the sequence: the same states bit for bit where the
    sequence is in one piece."""
    for ch, dtype in ((72, "bfloat16"), (35, "float32"), (64, "float16")):
        dev, val = make(torch, 5, 2000, 12, ch, dtype, "time", 0.1, True)
        op = gated_recurrence.GatedRecurrence(ch, dtype=getattr(torch, dtype))
        last = op.state(2000)
        y = op.sequence(dev["x"], dev["r"], dev["i"], dev["a"], reset=dev["reset"], state=dev["state"], state_out=last)
        state = dev["state"].clone()
        for t in range(12):
            out = op.step(dev["x"][:, t], dev["r"][:, t], dev["i"][:, t], dev["a"], state, done=dev["reset"][:, t])
            assert torch.equal(out, y[:, t]), t
        assert torch.equal(state, last)


@pytest.mark.parametrize("n,ch,dtype", [(1, 1, "float32"), (3, 7, "bfloat16"), (64, 1152, "bfloat16"), (1000, 330, "float16"),
                                        (5000, 36, "float32")])
def test_step(torch, n, ch, dtype):
    dev, val = make(torch, 3, n, 1, ch, dtype, "wide" if ch == 7 else "batch", 0.3, True)
    op = gated_recurrence.GatedRecurrence(ch, dtype=getattr(torch, dtype))
    out_state = op.state(n)
    y = op.step(dev["x"][:, 0], dev["r"][:, 0], dev["i"][:, 0], dev["a"], dev["state"], done=dev["reset"][:, 0], state_out=out_state)
    units, _ = bounds(val)
    want, last, _ = tr.recurrence(val["x"], val["r"], val["i"], val["a"], val["reset"], val["state"])
    near("y", y, want[:, 0], units["y"][:, 0], dtype)
    near("state", out_state, last, units["state"])


def test_resets_drop_what_was_there(torch):
    """NaN and infinity in the state and before an episode's start do not pass it, forward or backward."""
    for batch, time in ((600, 20), (1, 400)):
        dev, val = make(torch, 8, batch, time, 64, "float32", "batch", 0.0, True)
        reset = torch.zeros((batch, time), dtype=torch.bool, device="cuda")
        reset[:, 13] = True
        op = gated_recurrence.GatedRecurrence(64, dtype=torch.float32)
        four = lambda: (dev["x"], dev["r"], dev["i"], dev["a"])                            # noqa: E731
        saved = op.saved(batch, time)
        y = op.sequence(*four(), reset=reset, state=dev["state"], saved=saved)
        g = op.backward(dev["dy"], *four(), saved, reset=reset, want_dstate=True)
        dev["state"][:, 3] = float("nan")
        dev["x"][:, 5, 7] = float("inf")
        saved2 = op.saved(batch, time)
        y2 = op.sequence(*four(), reset=reset, state=dev["state"], saved=saved2)
        assert torch.equal(y2[:, 13:], y[:, 13:]) and torch.isnan(y2[:, 12, 3]).all() and torch.isinf(y2[:, 12, 7]).all()
        g2 = op.backward(dev["dy"], *four(), saved2, reset=reset, want_dstate=True)
        for key in ("dx", "dr", "di"):
            assert torch.equal(g2[key][:, 13:], g[key][:, 13:])
        # and what comes from behind the reset does not reach the steps before it
        dy = dev["dy"].clone()
        dy[:, 15, 20] = float("nan")
        g3 = op.backward(dy, dev["x"], dev["r"], dev["i"], dev["a"], saved, reset=reset, want_dstate=True)
        assert torch.isnan(g3["dx"][:, 13, 20]).all() and not torch.isnan(g3["dx"][:, :13, 20]).any()
        assert not torch.isnan(g3["dstate"][:, 20]).any()


def test_slow_channels_gather_no_bias(torch):
    """4,000 steps at decays of 0.999 and slower: independent roundings of at most u per operation, two a step, come to
    u sqrt(2 steps / 3) rms of what is kept; three times that is allowed."""
    time, ch = 4000, 512
    r = np.random.Generator(np.random.PCG64(0))
    a = -np.exp(r.uniform(np.log(1e-5), np.log(2e-3), ch)).astype(np.float32)
    op = gated_recurrence.GatedRecurrence(ch, dtype=torch.float32)
    x = np.zeros((1, time, ch), np.float32)
    gate = r.uniform(-1, 1, (1, time, ch)).astype(np.float32)
    state = r.uniform(1, 2, (1, ch)).astype(np.float32)
    d = lambda v: torch.from_numpy(v).cuda()                                               # noqa: E731
    last = op.state(1)
    op.sequence(d(x), d(gate), d(x), d(a), state=d(state), state_out=last)
    want = tr.recurrence(x, gate, x, a, state=state)[1]
    rel = f64(last) / want - 1.0
    assert np.sqrt((rel ** 2).mean()) <= 3 * U * np.sqrt(2 * time / 3.0)


def test_extreme_gates(torch):
    """Gates that vanish or saturate, a = 0 and large rates: finite, and the limits the header states."""
    op = gated_recurrence.GatedRecurrence(8, dtype=torch.float32)
    a = torch.tensor([0.0, -1e-30, -1e-6, -1.0, -50.0, -1e4, -0.0, -3e38], device="cuda")
    vals = [-3e38, -1e4, -90.0, -20.0, 0.0, 20.0, 90.0, 1e4, 3e38]
    r = torch.tensor(vals, device="cuda").repeat_interleave(len(vals)).view(-1, 1, 1).expand(-1, 6, 8).contiguous()
    i = torch.tensor(vals, device="cuda").repeat(len(vals)).view(-1, 1, 1).expand(-1, 6, 8).contiguous()
    x = torch.ones_like(r)
    n = r.shape[0]
    saved, last = op.saved(n, 6), op.state(n)
    y = op.sequence(x, r, i, a, state=torch.ones(n, 8, device="cuda"), state_out=last, saved=saved)
    g = op.backward(x, x, r, i, a, saved, want_dstate=True)
    for v in [y, last] + [g[k] for k in ("dx", "dr", "di", "dstate")]:
        assert torch.isfinite(v).all()
    assert (y[:, :, 0] == 1.0).all() and (g["dx"][:, :, 0] == 0.0).all()       # a = 0: nothing decays, nothing enters
    assert (y[r[:, 0, 0] < -100.0] == 1.0).all()                               # no gate, no decay
    assert (y[(r[:, 0, 0] > 10) & (i[:, 0, 0] > 50)][:, :, 5] == 1.0).all()    # all decays, all enters


@pytest.mark.parametrize("batch,time", [(1, 1), (2, 40), (1, 2000)])
def test_a_positive_rate_gives_nan_in_its_channel(torch, batch, time):
    op = gated_recurrence.GatedRecurrence(6, dtype=torch.float32)
    a = torch.tensor([-0.5, 0.5, -1.0, 30.0, 1e-3, -2.0], device="cuda")
    x = torch.ones((batch, time, 6), device="cuda")
    gate = torch.zeros_like(x)
    saved, last = op.saved(batch, time), op.state(batch)
    y = op.sequence(x, gate, gate, a, state_out=last, saved=saved)
    bad = a > 0
    g = op.backward(x, x, gate, gate, a, saved)
    for v in (y, last, g["dx"], g["dr"], g["di"], g["da"]):
        assert torch.isnan(v[..., bad]).all() and torch.isfinite(v[..., ~bad]).all()
    state = torch.zeros((batch, 6), device="cuda")
    one = op.step(x[:, 0], gate[:, 0], gate[:, 0], a, state)
    for v in (one, state):
        assert torch.isnan(v[..., bad]).all() and torch.isfinite(v[..., ~bad]).all()


def test_long_rows_beyond_32_bit_offsets(torch):
    batch, time, ch = 2, 3, 64
    stride = 2 ** 30 + 6
    dev, _ = make(torch, 4, batch, time, ch, "bfloat16")
    big = torch.empty((batch * time * stride // 1,), dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((batch, time, ch), (time * stride, stride, 1))
    op = gated_recurrence.GatedRecurrence(ch)
    want = op.sequence(dev["x"], dev["r"], dev["i"], dev["a"])
    far.copy_(dev["x"])
    got = op.sequence(far, dev["r"], dev["i"], dev["a"])
    assert torch.equal(got, want)
    op.sequence(dev["x"], dev["r"], dev["i"], dev["a"], out=far)
    assert torch.equal(far, want)


def test_side_stream_and_graph(torch):
    for batch, time in ((700, 24), (1, 500)):
        dev, _ = make(torch, 6, batch, time, 96, "bfloat16", "time", 0.05, True)
        op = gated_recurrence.GatedRecurrence(96)
        saved, last = op.saved(batch, time), op.state(batch)

        def run():
            y = op.sequence(dev["x"], dev["r"], dev["i"], dev["a"], reset=dev["reset"], state=dev["state"], state_out=last,
                            saved=saved)
            g = op.backward(dev["dy"], dev["x"], dev["r"], dev["i"], dev["a"], saved, reset=dev["reset"], want_dstate=True)
            return [y, last] + [g[k] for k in ("dx", "dr", "di", "da", "dstate")]

        want = [v.clone() for v in run()]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = run()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = run()
        dev["x"].mul_(0.5)
        graph.replay()
        first = [v.clone() for v in captured]
        assert all(torch.equal(p, q) for p, q in zip(first, run()))


def test_refusals(torch):
    op = gated_recurrence.GatedRecurrence(64)
    dev, _ = make(torch, 1, 4, 6, 64, "bfloat16", carry=True)
    x, r, i, a = (dev[k] for k in ("x", "r", "i", "a"))
    saved = op.saved(4, 6)
    for bad in (x.float(), x[:, :, :63], x.cpu(), x[:, :, ::2], x[:3]):
        with pytest.raises(ValueError):
            op.sequence(x, bad, i, a)
    for kw in (dict(state=dev["state"][:3]), dict(state_out=dev["state"].to(torch.bfloat16)), dict(saved=saved[1:]),
               dict(reset=torch.zeros(4, 6, device="cuda")), dict(out=x[:, :5])):
        with pytest.raises(ValueError):
            op.sequence(x, r, i, a, **kw)
    with pytest.raises(ValueError):
        op.sequence(x, r, i, a[:63])
    with pytest.raises(ValueError):
        op.step(x[:, 0], r[:, 0], i[:, 0], a, dev["state"].t())
    with pytest.raises(ValueError):
        op.backward(x, x, r, i, a, op.saved(4, 20))
    for call in (lambda: op.sequence(x[:0], r[:0], i[:0], a), lambda: op.sequence(x[:, :0], r[:, :0], i[:, :0], a),
                 lambda: op.sequence(x, r, i, a, out=x[:, :1].expand(4, 6, 64)),
                 lambda: op.sequence(x, r, i, a, state=dev["state"], state_out=dev["state"]),
                 lambda: op.step(x[:0, 0], r[:0, 0], i[:0, 0], a, dev["state"][:0])):
        with pytest.raises(gated_recurrence.GatedRecurrenceError) as ei:
            call()
        assert ei.value.code == -1
    for ch in (0, 65537):
        with pytest.raises(gated_recurrence.GatedRecurrenceError):
            gated_recurrence.GatedRecurrence(ch)
