"""The scan and the convolution over the loops that large calls run in: many steps, several chunks per
segment, several rows per block, whole vectors.  Cases state how their work is cut (test_host_calls.py holds
the libraries to it), so that a change of the cut cannot leave a loop without a test.

Tolerances of the scan.  One unit is 2^-23 relative.  Results of the exponential, reciprocal and the series of
softplus are taken within 2 units each; with the rounding of its argument v the step delta is then within
e = 8 + |v| units, the gate within 8 + |z|, and a decay exp(delta A) within

    r = 2 + |delta A| (2 + e + L) units,

where L, the steps of a segment, stands for the sum of deltas by which segments are joined (0 where the
time axis is not cut).  With H the state over absolute values, an error bound E of the state follows the
recurrence itself, so that it is forgotten as the state is:

    E_t = decay E_{t-1} + 2^-23 (r decay H_{t-1} + (e + 2) |delta x b| + H_t)

and likewise backwards for dh and what arrives from later steps.  A sum of K terms adds K units of its
absolute terms, where K is the longest chain of additions that an order of the sum has.  Every result is
rounded once to its type.  A tenth is added for second-order terms.
"""
import numpy as np
import pytest

from oracle import sequence as seq
from paper_2603_12145_b200 import ssm

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -23
UNIT = {"float32": 2.0 ** -23, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}

# batch, time, channels, states, groups, dtype, time-major, and the cut: segments and chunks per segment forward,
# segments, chunks per segment and blocks per tile of channels backward
SCAN = [
    (700, 40, 33, 16, 1, "float32", False, (1, 3), (1, 3, 700)),       # rows alone fill the device
    (100, 40, 66, 16, 33, "float32", True, (1, 3), (1, 3, 34)),        # three rows per block backward
    (600, 20, 66, 16, 33, "bfloat16", True, (1, 2), (1, 2, 36)),       # seventeen rows per block
    (620, 33, 130, 4, 1, "bfloat16", False, (1, 3), (1, 3, 310)),      # two rows, several tiles of channels
    (90, 40, 66, 24, 33, "float32", False, (1, 3), (1, 3, 30)),        # two blocks of 16 states
    (80, 35, 44, 48, 22, "float16", True, (1, 3), (1, 3, 40)),         # four
    (1, 600, 33, 16, 33, "float32", False, (13, 3), (8, 5, 8)),        # segments of several chunks
    (2, 400, 22, 24, 22, "float32", True, (9, 3), (13, 2, 26)),
    (1, 500, 34, 64, 17, "bfloat16", False, (16, 2), (8, 4, 8)),
    (300, 100, 35, 5, 1, "float16", True, (1, 7), (1, 7, 300)),
]
# rows, channels, states, groups, dtype; and rows of a block, which takes them four at a time
STEPS = [
    (3001, 129, 16, 1, "bfloat16", 8), (2000, 260, 16, 2, "float32", 9), (1500, 70, 8, 1, "float16", 4),
    (5000, 515, 4, 1, "float32", 13), (1201, 36, 32, 1, "bfloat16", 4), (3000, 40, 64, 2, "float16", 8), (900, 66, 24, 3, "float32", 4),
]
# batch, time, channels, width, dtype, time-major; and the steps of a run, runs of a warp backward
CONV = [
    (1200, 130, 36, 4, "bfloat16", True, 32, 3), (1200, 100, 36, 3, "float16", False, 32, 3), (1300, 70, 20, 4, "float32", True, 16, 3),
    (4800, 129, 8, 2, "float16", False, 128, 5), (2400, 65, 8, 4, "float16", True, 64, 3), (900, 50, 35, 4, "bfloat16", True, 8, 3),
]


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    ssm.load(build_if_missing=True)
    return torch


def test_a_slow_state_does_not_drift(torch):
    """1,000 steps without input of states that keep about 0.999 per step, as one sequence and as single
    tokens.

    Tolerance, in units of 2^-23 relative, for the mean over 614,400 states (what is random averages out: a
    rounding per step, below 1 unit, over sqrt(1000 * 614,400) of them).  What the kernels leave of the
    exponential's own bias (measured between 0.05 and 0.22 units low, depending on the argument; they take out a
    constant) is to stay below 0.15 per step; the rate's and the steps' own roundings scale the exponent, which is about 1, by a few units.  The
    two forms are the same recurrence and may differ by a twentieth of a unit per step, a quarter of that bias,
    which a form that does not take it out would show in full."""
    steps, rows, ch, n = 1000, 300, 128, 16
    r = np.random.Generator(np.random.PCG64(1))
    a = -np.exp(0.2 * r.standard_normal((ch, n)))
    dt = np.log(np.expm1(1e-3 * np.exp(0.2 * r.standard_normal((rows, 1, ch)))))
    h0 = r.uniform(0.5, 1.0, (rows, ch, n))
    a, dt, h0 = [torch.from_numpy(v.astype(np.float32)).cuda() for v in (a, dt, h0)]
    delta = torch.nn.functional.softplus(dt[:, 0].double())
    want = h0.double() * torch.exp(steps * delta.unsqueeze(2) * a.double())
    op = ssm.Ssm(ch, n, dtype=torch.float32)
    assert op._lib.ssm_scan_workspace_bytes(op.h, rows, steps, 0) == 0       # not cut along the time axis
    zero, ones = torch.zeros((rows, steps, ch), device="cuda"), torch.ones((rows, steps, n), device="cuda")
    whole = op.state(rows)
    op.scan(zero, dt.expand(rows, steps, ch), a, ones, ones, state=h0, state_out=whole)
    stepped = h0.clone()
    for _ in range(steps):
        op.scan_step(zero[:, 0], dt[:, 0], a, ones[:, 0], ones[:, 0], stepped)
    drift = [((h.double() / want - 1).mean() / EPS).item() for h in (stepped, whole)]
    assert abs(drift[0] - drift[1]) <= 0.05 * steps, drift
    assert max(abs(d) for d in drift) <= 0.15 * steps + 4, drift


def tensor(torch, a, dtype="float32", time_major=False):
    """(device tensor, its values as binary64)."""
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda().to(getattr(torch, dtype))
    if time_major:
        t = t.transpose(0, 1).contiguous().transpose(0, 1)
    return t, t.double().cpu().numpy()


def check(name, got, want, tol, dtype="float32"):
    got = got.double().cpu().numpy()
    tol = 1.1 * tol + UNIT[dtype] * np.abs(want) + (2.0 ** -24 if dtype == "float16" else 1e-30)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, first at %s: got %r want %r tol %r" % (
        name, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], np.broadcast_to(tol, got.shape)[bad][0])


def scan_bounds(v, groups, segment, chain, back_segment):
    """Error bounds of all outputs of a scan and its gradients (the rules above).  segment, back_segment: L of the two
    directions; chain: additions behind one parameter's gradient."""
    x, dt, b, c, z, dy = [np.abs(v[k]) if k != "dt" else v[k] for k in ("x", "dt", "b", "c", "z", "dy")]
    a, d, bias = np.abs(v["a"]), np.abs(v["d"]), v["dt_bias"]
    batch, time, ch = x.shape
    n, per = a.shape[1], ch // groups
    out = {k: np.zeros_like(x) for k in ("y", "dx", "ddt", "dz")}
    out.update({k: np.zeros((batch, time, groups * n)) for k in ("db", "dc")})
    out.update(da=np.zeros_like(a), dd=np.zeros(ch), ddt_bias=np.zeros(ch))
    wide = lambda u: np.repeat(u.reshape(batch, groups, n), per, axis=1)                     # noqa: E731
    by_group = lambda u: u.reshape(batch, groups, per, n).sum(axis=2).reshape(batch, -1)     # noqa: E731
    kept = []
    h, err = np.abs(v["state"]), np.zeros((batch, ch, n))

    def step(t, length):
        raw = dt[:, t] + bias
        delta = np.logaddexp(0.0, raw)
        e = 8 + np.abs(raw)
        decay = np.exp(-delta[:, :, None] * a)
        return raw, delta, e, decay, 2 + delta[:, :, None] * a * (2 + e[:, :, None] + length)

    def start(t):
        return (v["reset"][:, t] != 0)[:, None, None]

    for t in range(time):
        raw, delta, e, decay, r = step(t, segment)
        h, err = np.where(start(t), 0.0, h), np.where(start(t), 0.0, err)
        kept.append((h, err))
        into = (delta * x[:, t])[:, :, None] * wide(b[:, t])
        before, h = h, decay * h + into
        err = decay * err + EPS * (r * decay * before + (e[:, :, None] + 2) * into + h)
        gate = z[:, t] * seq.sigmoid(v["z"][:, t])
        mag = (wide(c[:, t]) * h).sum(axis=2) + d * x[:, t]
        out["y"][:, t] = gate * ((wide(c[:, t]) * err).sum(axis=2) + EPS * (n + 12 + z[:, t]) * mag)
    out["state"] = err
    arrives, arrives_err = np.abs(v["dstate_out"]), np.zeros_like(h)
    for t in range(time - 1, -1, -1):
        raw, delta, e, decay, r = step(t, back_segment)
        before, before_err = kept[t]
        bt, ct, e3 = wide(b[:, t]), wide(c[:, t]), e[:, :, None]
        into = (delta * x[:, t])[:, :, None] * bt
        ah = decay * before
        ah_err = decay * before_err + EPS * (r + 1) * ah
        h, h_err = ah + into, ah_err + EPS * ((e3 + 2) * into + ah + into)
        rg = 10 + z[:, t]
        g = dy[:, t] * z[:, t] * seq.sigmoid(v["z"][:, t])
        slope = seq.dsilu(v["z"][:, t], magnitude=True)
        mag = (ct * h).sum(axis=2) + d * x[:, t]
        out["dz"][:, t] = dy[:, t] * slope * ((ct * h_err).sum(axis=2) + EPS * (n + 3 + rg + 2) * mag)
        dh = arrives + g[:, :, None] * ct
        dh_err = arrives_err + EPS * (rg[:, :, None] * g[:, :, None] * ct + dh)
        out["dc"][:, t] = by_group(g[:, :, None] * (h_err + EPS * (rg[:, :, None] + per) * h))
        out["db"][:, t] = by_group((delta * x[:, t])[:, :, None] * (dh_err + EPS * (e3 + 2 + per) * dh))
        pull = (dh * bt).sum(axis=2)
        pull_err = (dh_err * bt).sum(axis=2) + EPS * (n + 2) * pull
        out["dx"][:, t] = EPS * (rg + 2) * d * g + delta * (pull_err + EPS * (e + 2) * pull)
        qq, qq_err = dh * ah, dh_err * ah + dh * ah_err + EPS * dh * ah
        s, s_err = (a * qq).sum(axis=2), (a * (qq_err + EPS * (n + 3) * qq)).sum(axis=2)
        sig = seq.sigmoid(raw)
        ddt = (s + x[:, t] * pull) * sig
        ddt_err = (s_err + x[:, t] * pull_err) * sig + EPS * (12 + np.abs(raw)) * ddt
        out["ddt"][:, t] = ddt_err
        out["ddt_bias"] += (ddt_err + EPS * chain * ddt).sum(axis=0)
        out["dd"] += (EPS * (rg + 1 + chain) * g * x[:, t]).sum(axis=0)
        out["da"] += (delta[:, :, None] * (qq_err + EPS * (e3 + 1 + chain) * qq)).sum(axis=0)
        arrives_err = np.where(start(t), 0.0, decay * (dh_err + EPS * (r + 1) * dh))
        arrives = np.where(start(t), 0.0, decay * dh)
    out["dstate"] = arrives_err
    return out


@pytest.mark.parametrize("case", SCAN, ids=str)
def test_scan_and_gradients(torch, case):
    batch, time, ch, n, groups, dtype, time_major, forward_cut, backward_cut = case
    r = np.random.Generator(np.random.PCG64(batch + time))
    dev, val = {}, {}
    for name, feat, scale in (("x", ch, 1.0), ("dt", ch, 0.7), ("b", groups * n, 1.0), ("c", groups * n, 1.0),
                              ("z", ch, 1.0), ("dy", ch, 1.0)):
        dev[name], val[name] = tensor(torch, scale * r.standard_normal((batch, time, feat)), dtype, time_major)
    for name, v in (("a", -np.exp(0.7 * r.standard_normal((ch, n)))), ("d", 1 + 0.3 * r.standard_normal(ch)),
                    ("dt_bias", r.uniform(-6.0, -1.0, ch)), ("state", r.standard_normal((batch, ch, n))),
                    ("dstate_out", r.standard_normal((batch, ch, n)))):
        dev[name], val[name] = tensor(torch, v)
    val["reset"] = (r.random((batch, time)) < 0.03).astype(np.uint8)
    dev["reset"] = torch.from_numpy(val["reset"]).cuda()
    segment, back_segment = [16 * c[1] if c[0] > 1 else 0 for c in (forward_cut, backward_cut)]
    rows_of_a_block = -(-batch * backward_cut[0] // backward_cut[2])
    chain = rows_of_a_block * min(time, 16 * backward_cut[1]) + backward_cut[2] // 8 + 8
    tol = scan_bounds(val, groups, segment, chain, back_segment)
    inputs = {k: val[k] for k in ("x", "dt", "a", "b", "c", "d", "z", "dt_bias", "reset", "state")}
    want = dict(zip(("y", "state"), seq.scan(groups=groups, **inputs)))
    op = ssm.Ssm(ch, n, groups, dtype=getattr(torch, dtype))
    saved, state = op.saved(batch, time), op.state(batch)
    args = {k: dev[k] for k in ("d", "z", "dt_bias", "reset")}
    first = [dev[k] for k in ("x", "dt", "a", "b", "c")]
    got = {"y": op.scan(*first, state=dev["state"], state_out=state, saved=saved, **args), "state": state}
    check("y", got["y"], want["y"], tol["y"], dtype)
    check("state", got["state"], want["state"], tol["state"])
    want = seq.scan_grad(val["dy"], dstate_out=val["dstate_out"], groups=groups, **inputs)
    got = op.scan_backward(dev["dy"], *first, saved, dstate_out=dev["dstate_out"], want_dstate=True, **args)
    for key in ("dx", "ddt", "dz", "db", "dc"):
        check(key, got[key], want[key], tol[key], dtype)
    for key in ("da", "dd", "ddt_bias", "dstate"):
        check(key, got[key], want[key], tol[key])
    again = op.scan_backward(dev["dy"], *first, saved, dstate_out=dev["dstate_out"], want_dstate=True, **args)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("case", STEPS, ids=str)
def test_scan_step_on_whole_vectors(torch, case):
    """Contiguous rows, so that states, b and c come in whole vectors, and rows enough for several turns of a block."""
    n, ch, states, groups, dtype, _ = case
    r = np.random.Generator(np.random.PCG64(n))
    dev, val = {}, {}
    for name, feat in (("x", ch), ("dt", ch), ("b", groups * states), ("c", groups * states), ("z", ch)):
        dev[name], val[name] = tensor(torch, r.standard_normal((n, 1, feat)), dtype)
    for name, v in (("a", -np.exp(0.7 * r.standard_normal((ch, states)))), ("d", 1 + 0.3 * r.standard_normal(ch)),
                    ("dt_bias", r.uniform(-6.0, -1.0, ch)), ("state", r.standard_normal((n, ch, states)))):
        dev[name], val[name] = tensor(torch, v)
    val["reset"] = (r.random((n, 1)) < 0.2).astype(np.uint8)
    done = torch.from_numpy(val["reset"][:, 0].copy()).cuda()
    inputs = {k: val[k] for k in ("x", "dt", "a", "b", "c", "d", "z", "dt_bias", "reset", "state")}
    want_y, want_h = seq.scan(groups=groups, **inputs)
    tol = scan_bounds({**val, "dy": val["x"], "dstate_out": 0 * val["state"]}, groups, 0, 0, 0)
    op = ssm.Ssm(ch, states, groups, dtype=getattr(torch, dtype))
    row = {k: dev[k][:, 0] for k in ("x", "dt", "b", "c", "z")}
    assert row["b"].stride(0) % 4 == 0 and row["b"].data_ptr() % 16 == 0
    y = op.scan_step(row["x"], row["dt"], dev["a"], row["b"], row["c"], dev["state"], d=dev["d"], z=row["z"],
                     dt_bias=dev["dt_bias"], done=done)
    check("y", y, want_y[:, 0], tol["y"][:, 0], dtype)
    check("state", dev["state"], want_h, tol["state"])


@pytest.mark.parametrize("case", CONV, ids=str)
def test_conv_and_gradients(torch, case):
    """As in test_gpu_ssm.py: width + 1 roundings of the sum, 8 of the activation; a parameter's gradient adds the longest
    chain of its sum: the steps of a warp's runs, then an eighth of the warps and eight."""
    batch, time, ch, width, dtype, time_major, run, runs = case
    r = np.random.Generator(np.random.PCG64(batch))
    dev, val = {}, {}
    for name in ("x", "dy"):
        dev[name], val[name] = tensor(torch, r.standard_normal((batch, time, ch)), dtype, time_major)
    for name, shape, kind in (("w", (ch, width), "float32"), ("bias", (ch,), "float32"), ("history", (batch, width - 1, ch), dtype)):
        dev[name], val[name] = tensor(torch, r.standard_normal(shape), kind)
    val["reset"] = (r.random((batch, time)) < 0.05).astype(np.uint8)
    dev["reset"] = torch.from_numpy(val["reset"]).cuda()
    keys = ("x", "w", "bias", "reset", "history")
    inputs = {k: val[k] for k in keys}
    want_y, want_h = seq.conv(**inputs)
    mag_y, _ = seq.conv(magnitude=True, **inputs)
    op = ssm.Ssm(ch, width=width, dtype=getattr(torch, dtype))
    history = op.history(batch)
    y = op.conv(*[dev[k] for k in keys], history_out=history)
    factor = width + 9
    check("y", y, want_y, EPS * factor * 1.1 * mag_y, dtype)
    assert np.array_equal(history.double().cpu().numpy(), want_h)
    want = seq.conv_grad(val["dy"], **inputs)
    mag = seq.conv_grad(val["dy"], magnitude=True, **inputs)
    got = op.conv_backward(dev["dy"], *[dev[k] for k in keys])
    chain = run * runs + batch * -(-time // run) // runs // 8 + 8
    for name, g, w, m, extra, kind in zip(("dx", "dw", "dbias"), got, want, mag, (width, chain, chain), (dtype, "float32", "float32")):
        check(name, g, w, EPS * (factor + extra) * m, kind)
    for t in range(3):
        step = op.conv_step(dev["x"][:, t].contiguous(), dev["history"], dev["w"], dev["bias"], done=dev["reset"][:, t])
        check("step %d" % t, step, want_y[:, t], EPS * factor * 1.1 * mag_y[:, t], dtype)


@pytest.mark.parametrize("rows,dtype", [(300, "float32"), (1, "bfloat16")])
def test_steps_of_no_length_leave_the_state_as_it_is(torch, rows, dtype):
    """delta = softplus(-inf) = 0: the state's bits do not change over 1,000 steps, neither as one sequence (uncut, and cut
    along the time axis) nor as single tokens; nor does a gradient on its way back, and none reaches dt or A."""
    steps, ch, n = 1000, 128, 16
    kind = getattr(torch, dtype)
    gen = torch.Generator("cuda").manual_seed(2)
    draw = lambda *s: torch.randn(s, device="cuda", generator=gen)      # noqa: E731
    op = ssm.Ssm(ch, n, dtype=kind)
    assert (op._lib.ssm_scan_workspace_bytes(op.h, rows, steps, 0) == 0) == (rows == 300)
    a, h0, x, b = -torch.exp(draw(ch, n)), draw(rows, ch, n), draw(rows, steps, ch).to(kind), draw(rows, steps, n).to(kind)
    still, out = torch.full((rows, steps, ch), -float("inf"), dtype=kind, device="cuda"), op.state(rows)
    op.scan(x, still, a, b, b, state=h0, state_out=out)
    assert torch.equal(out, h0)
    for t in range(steps):
        op.scan_step(x[:, t], still[:, t], a, b[:, t], b[:, t], out)
    assert torch.equal(out, h0)
    saved = op.saved(rows, steps)
    op.scan(x, still, a, b, b, state=h0, saved=saved)
    dy = torch.zeros_like(x)
    d0 = draw(rows, ch, n)
    got = op.scan_backward(dy, x, still, a, b, b, saved, dstate_out=d0, want_dstate=True)
    assert torch.equal(got["dstate"], d0) and bool((got["ddt"] == 0).all()) and bool((got["da"] == 0).all())
