"""Binary64 definitions of the sequence operators (causal convolution, selective scan, gated
feed-forward block) in numpy, one time step after the other -- TEST INFRASTRUCTURE: only tests,
the smoke check and the benchmark's CPU legs may import it.

Every function takes `magnitude`: the same sums with every term replaced by its absolute value,
which is what rounding errors are measured against."""
from __future__ import annotations

import numpy as np


def sigmoid(v):
    return np.exp(-np.logaddexp(0.0, -v))


def silu(v):
    return v * sigmoid(v)


def dsilu(v, magnitude=False):
    s = sigmoid(v)
    return s + (np.abs(v) if magnitude else v) * s * (1.0 - s)


def gelu(v):
    return 0.5 * v * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (v + 0.044715 * v ** 3)))


def dgelu(v):
    c = np.sqrt(2.0 / np.pi)
    t = np.tanh(c * (v + 0.044715 * v ** 3))
    return 0.5 * (1.0 + t) + 0.5 * v * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * v * v)


ACTIVATIONS = {"silu": (silu, dsilu), "gelu": (gelu, dgelu)}


def _f(*arrays):
    return [None if a is None else np.asarray(a, dtype=np.float64) for a in arrays]


def _conv_windows(x, reset, history, width):
    """Yields (t, taps [batch, width, channels], age [batch]): the inputs that step t sees, oldest
    first, and how many steps ago its episode began (large if before the sequence)."""
    batch, time, ch = x.shape
    window = np.zeros((batch, width - 1, ch)) if history is None else history.copy()
    age = np.full(batch, width)
    for t in range(time):
        age = age + 1
        if reset is not None:
            hit = np.asarray(reset)[:, t] != 0
            window[hit] = 0.0
            age = np.where(hit, 0, age)
        taps = np.concatenate([window, x[:, t:t + 1]], axis=1)
        yield t, taps, age
        window = taps[:, 1:].copy()


def conv(x, w, bias=None, reset=None, history=None, magnitude=False):
    """(y, history after the last step)."""
    x, w, bias, history = _f(x, w, bias, history)
    y = np.empty_like(x)
    bias = np.zeros(x.shape[2]) if bias is None else bias
    for t, taps, _ in _conv_windows(x, reset, history, w.shape[1]):
        if magnitude:
            # |silu(u + e) - silu(u)| <= 1.1 |e|
            y[:, t] = np.abs(bias) + (np.abs(taps) * np.abs(w.T)).sum(axis=1)
        else:
            y[:, t] = silu(bias + (taps * w.T).sum(axis=1))
    return y, taps[:, 1:]


def conv_grad(dy, x, w, bias=None, reset=None, history=None, magnitude=False):
    """(dx, dw, dbias)."""
    dy, x, w, bias, history = _f(dy, x, w, bias, history)
    width = w.shape[1]
    b0 = np.zeros(x.shape[2]) if bias is None else bias
    dx, dw, dbias = np.zeros_like(x), np.zeros_like(w), np.zeros(x.shape[2])
    wa = np.abs(w) if magnitude else w
    for t, taps, age in _conv_windows(x, reset, history, width):
        u = b0 + (taps * w.T).sum(axis=1)
        if magnitude:
            # an error e of u moves the slope by at most |e| / 2
            mag = np.abs(b0) + (np.abs(taps) * np.abs(w.T)).sum(axis=1)
            dpre, taps = np.abs(dy[:, t]) * (1.1 + mag), np.abs(taps)
        else:
            dpre = dy[:, t] * dsilu(u)
        dbias += dpre.sum(axis=0)
        dw += (taps * dpre[:, None]).sum(axis=0).T
        for j in range(min(width, t + 1)):
            dx[:, t - j] += np.where((age >= j)[:, None], dpre * wa[:, width - 1 - j], 0.0)
    return dx, dw, dbias


def _per_channel(v, groups, channels):
    """[batch, groups * states] -> [batch, channels, states]: a channel sees its group's row."""
    batch = v.shape[0]
    return np.repeat(v.reshape(batch, groups, -1), channels // groups, axis=1)


def scan(x, dt, a, b, c, d=None, z=None, dt_bias=None, reset=None, state=None, groups=1, magnitude=False,
         keep=None):
    """(y, state after the last step).  keep: a list that receives the state before every step
    (after the reset)."""
    x, dt, a, b, c, d, z, dt_bias, state = _f(x, dt, a, b, c, d, z, dt_bias, state)
    batch, time, ch = x.shape
    if magnitude:
        x, b, c, d, state = [None if v is None else np.abs(v) for v in (x, b, c, d, state)]
    h = np.zeros((batch, ch, a.shape[1])) if state is None else state.copy()
    y = np.empty_like(x)
    for t in range(time):
        if reset is not None:
            h = np.where((np.asarray(reset)[:, t] != 0)[:, None, None], 0.0, h)
        if keep is not None:
            keep.append(h)
        delta = np.logaddexp(0.0, dt[:, t] + (0.0 if dt_bias is None else dt_bias))
        h = np.exp(delta[:, :, None] * a) * h + (delta * x[:, t])[:, :, None] * _per_channel(b[:, t], groups, ch)
        y[:, t] = (_per_channel(c[:, t], groups, ch) * h).sum(axis=2)
        if d is not None:
            y[:, t] += d * x[:, t]
        if z is not None:
            y[:, t] *= np.abs(silu(z[:, t])) if magnitude else silu(z[:, t])
    return y, h


def scan_grad(dy, x, dt, a, b, c, d=None, z=None, dt_bias=None, reset=None, state=None, dstate_out=None, groups=1,
              magnitude=False):
    """Gradients as a dict: dx, ddt, da, db, dc, dd, dz, ddt_bias, dstate."""
    before = []
    scan(x, dt, a, b, c, d, z, dt_bias, reset, state, groups, magnitude, before)
    dy, x, dt, a, b, c, d, z, dt_bias, dstate_out = _f(dy, x, dt, a, b, c, d, z, dt_bias, dstate_out)
    rate = a
    if magnitude:
        dy, x, b, c, d, rate, dstate_out = [None if v is None else np.abs(v) for v in (dy, x, b, c, d, a, dstate_out)]
    batch, time, ch = x.shape
    n = a.shape[1]
    out = {"dx": np.empty_like(x), "ddt": np.empty_like(x), "dz": np.zeros_like(x), "da": np.zeros_like(a),
           "db": np.empty((batch, time, groups * n)), "dc": np.empty((batch, time, groups * n)),
           "dd": np.zeros(ch), "ddt_bias": np.zeros(ch)}
    skip = np.zeros(ch) if d is None else d
    carry = np.zeros((batch, ch, n)) if dstate_out is None else dstate_out.copy()

    def by_group(v):     # [batch, channels, states] -> sum over the group's channels
        return v.reshape(batch, groups, ch // groups, n).sum(axis=2).reshape(batch, groups * n)

    for t in range(time - 1, -1, -1):
        raw = dt[:, t] + (0.0 if dt_bias is None else dt_bias)
        delta = np.logaddexp(0.0, raw)
        bt, ct = _per_channel(b[:, t], groups, ch), _per_channel(c[:, t], groups, ch)
        decay = np.exp(delta[:, :, None] * a)
        into = decay * before[t]
        h = into + (delta * x[:, t])[:, :, None] * bt
        g = dy[:, t]
        if z is not None:
            f, df = silu(z[:, t]), dsilu(z[:, t], magnitude)
            if magnitude:
                f = np.abs(f)
            out["dz"][:, t] = g * ((ct * h).sum(axis=2) + skip * x[:, t]) * df
            g = g * f
        dh = carry + g[:, :, None] * ct
        out["dc"][:, t] = by_group(g[:, :, None] * h)
        out["db"][:, t] = by_group(dh * (delta * x[:, t])[:, :, None])
        pull = (dh * bt).sum(axis=2)
        out["dx"][:, t] = skip * g + delta * pull
        ddt = ((dh * into * rate).sum(axis=2) + x[:, t] * pull) * sigmoid(raw)
        out["ddt"][:, t] = ddt
        out["ddt_bias"] += ddt.sum(axis=0)
        out["dd"] += (g * x[:, t]).sum(axis=0)
        out["da"] += (dh * into * delta[:, :, None]).sum(axis=0)
        carry = decay * dh
        if reset is not None:
            carry = np.where((np.asarray(reset)[:, t] != 0)[:, None, None], 0.0, carry)
    out["dstate"] = carry
    return out


def gated_ffn(x, w_in, w_out, activation="silu"):
    """(y, pre-activations [n, 2 hidden], hidden)."""
    x, w_in, w_out = _f(x, w_in, w_out)
    act, _ = ACTIVATIONS[activation]
    f = w_out.shape[1]
    pre = x @ w_in.T
    hidden = act(pre[:, :f]) * pre[:, f:]
    return hidden @ w_out.T, pre, hidden


def gated_ffn_grad(dy, x, w_in, w_out, activation="silu"):
    """(dx, dw_in, dw_out)."""
    dy, x, w_in, w_out = _f(dy, x, w_in, w_out)
    act, slope = ACTIVATIONS[activation]
    f = w_out.shape[1]
    _, pre, hidden = gated_ffn(x, w_in, w_out, activation)
    dh = dy @ w_out
    dpre = np.concatenate([dh * pre[:, f:] * slope(pre[:, :f]), dh * act(pre[:, :f])], axis=1)
    return dpre @ w_in, dpre.T @ x, dy.T @ hidden
