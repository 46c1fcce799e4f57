"""Binary64 definitions of the operators of a policy's training step (layer norm with the residual stream, gated linear
recurrence, orthogonalised update) in numpy -- TEST INFRASTRUCTURE: only tests and the smoke check may import it."""
from __future__ import annotations

import numpy as np


def _f(*arrays):
    return [None if a is None else np.asarray(a, dtype=np.float64) for a in arrays]


def sigmoid(v):
    return np.exp(-np.logaddexp(0.0, -v))


# ---- layer norm ---------------------------------------------------------------------

def norm(s, w=None, b=None, eps=1e-5):
    """(y, mean, 1 / standard deviation) of the rows s [n, width]."""
    s, w, b = _f(s, w, b)
    mean = s.mean(axis=1)
    scale = 1.0 / np.sqrt(((s - mean[:, None]) ** 2).mean(axis=1) + eps)
    y = (s - mean[:, None]) * scale[:, None]
    if w is not None:
        y = y * w
    if b is not None:
        y = y + b
    return y, mean, scale


def norm_grad(dy, s, w=None, dsum=None, eps=1e-5):
    """(dx, dw, db)."""
    dy, s, w, dsum = _f(dy, s, w, dsum)
    _, mean, scale = norm(s, eps=eps)
    z = (s - mean[:, None]) * scale[:, None]
    c = dy if w is None else dy * w
    dx = scale[:, None] * (c - c.mean(axis=1, keepdims=True) - z * (c * z).mean(axis=1, keepdims=True))
    if dsum is not None:
        dx = dx + dsum
    return dx, (dy * z).sum(axis=0), dy.sum(axis=0)


# ---- gated linear recurrence --------------------------------------------------------

def recurrence(x, r, i, a, reset=None, state=None):
    """(y, last state, states before each step) of sequences [batch, time, channels], one step after the other."""
    x, r, i, a, state = _f(x, r, i, a, state)
    batch, time, ch = x.shape
    h = np.zeros((batch, ch)) if state is None else state.copy()
    y, before = np.empty_like(x), np.empty_like(x)
    for t in range(time):
        if reset is not None:
            h = np.where(np.asarray(reset)[:, t, None] != 0, 0.0, h)
        before[:, t] = h
        rate = a * sigmoid(r[:, t])
        h = np.exp(rate) * h + np.sqrt(-np.expm1(2.0 * rate)) * sigmoid(i[:, t]) * x[:, t]
        y[:, t] = h
    return y, h, before


def recurrence_grad(dy, x, r, i, a, reset=None, state=None, dstate_out=None, magnitude=False):
    """Gradients as a dict (dx, dr, di, da, dstate).  magnitude: every term by its absolute value.  Where a channel's
    decay is exactly one (a = 0, or a gate that has vanished), its rate's derivative has no limit and counts as zero."""
    before = recurrence(x, r, i, a, reset, state)[2]
    dy, x, r, i, a, dstate_out = _f(dy, x, r, i, a, dstate_out)
    if magnitude:
        dy, x = np.abs(dy), np.abs(x)
        before = recurrence(x, r, i, a, reset, None if state is None else np.abs(np.asarray(state, dtype=np.float64)))[2]
        dstate_out = None if dstate_out is None else np.abs(dstate_out)
    batch, time, ch = x.shape
    out = {k: np.empty_like(x) for k in ("dx", "dr", "di")}
    out["da"] = np.zeros(ch)
    g = np.zeros((batch, ch)) if dstate_out is None else dstate_out.copy()
    sign = 1.0 if magnitude else -1.0
    for t in range(time - 1, -1, -1):
        g = g + dy[:, t]
        sr, si = sigmoid(r[:, t]), sigmoid(i[:, t])
        rate = a * sr
        decay, gain = np.exp(rate), np.sqrt(-np.expm1(2.0 * rate))
        slope = np.divide(1.0, gain, out=np.zeros_like(gain), where=gain > 0)
        drate = g * (before[:, t] * decay + sign * si * x[:, t] * decay ** 2 * slope)
        out["dx"][:, t] = g * gain * si
        out["di"][:, t] = g * gain * x[:, t] * si * (1.0 - si)
        out["dr"][:, t] = drate * (np.abs(rate) if magnitude else rate) * (1.0 - sr)
        out["da"] += (drate * sr).sum(axis=0)
        g = g * decay
        if reset is not None:
            g = np.where(np.asarray(reset)[:, t, None] != 0, 0.0, g)
    out["dstate"] = g
    return out


# ---- orthogonalised update ----------------------------------------------------------

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def orthogonal(g, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """The update of one matrix [rows, cols]: p(p(...p(X))) with X = g / (|g| + eps), p(X) = a X + (b A + c A^2) X, A = X X^T."""
    a, b, c = coefficients
    x = np.asarray(g, dtype=np.float64)
    x = x / (np.sqrt((x * x).sum()) + eps)
    for _ in range(steps):
        if x.shape[0] <= x.shape[1]:
            gram = x @ x.T
            x = a * x + (b * gram + c * gram @ gram) @ x
        else:
            gram = x.T @ x
            x = a * x + x @ (b * gram + c * gram @ gram)
    return x
