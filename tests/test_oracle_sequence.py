"""Pins of the binary64 sequence oracle: hand-computed cases, gradients against central
differences, and the operators' own invariances (cutting a sequence, resets, token by token)."""
import numpy as np
import pytest

from oracle import sequence as seq


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def test_conv_by_hand():
    x = np.array([[[1.0], [2.0], [-1.0], [3.0]]])
    w = np.array([[10.0, 100.0, 1000.0]])
    u = [1000.0, 2000.0 + 100.0, -1000.0 + 200.0 + 10.0, 3000.0 - 100.0 + 20.0]
    y, hist = seq.conv(x, w)
    assert np.allclose(y[0, :, 0], [seq.silu(np.float64(v)) for v in u])
    assert np.array_equal(hist[0, :, 0], [-1.0, 3.0])
    # a reset at step 2 drops the taps from before it, also for the steps after
    y, hist = seq.conv(x, w, reset=np.array([[0, 0, 1, 0]]))
    u = [1000.0, 2100.0, -1000.0, 3000.0 - 100.0]
    assert np.allclose(y[0, :, 0], [seq.silu(np.float64(v)) for v in u])
    y, hist = seq.conv(x[:, :1], w, reset=np.array([[1]]), history=np.full((1, 2, 1), 7.0))
    assert np.allclose(y[0, 0, 0], 1000.0) and np.array_equal(hist[0, :, 0], [0.0, 1.0])


def test_scan_by_hand():
    # one channel, one state, delta = log 2 (dt = 0): a = -1 halves the state per step
    x = np.array([[[1.0], [0.0], [2.0]]])
    ones = np.ones((1, 3, 1))
    ln2 = np.log(2.0)
    y, h = seq.scan(x, np.zeros((1, 3, 1)), np.array([[-1.0]]), ones, 3.0 * ones, d=np.array([5.0]))
    hs = [ln2, ln2 / 2, ln2 / 4 + 2 * ln2]
    assert np.allclose(y[0, :, 0], [3 * hs[0] + 5, 3 * hs[1], 3 * hs[2] + 10]) and np.allclose(h[0, 0, 0], hs[2])
    y, h = seq.scan(x, np.zeros((1, 3, 1)), np.array([[-1.0]]), ones, ones, reset=np.array([[0, 0, 1]]),
                    state=np.full((1, 1, 1), 8.0))
    assert np.allclose(y[0, :, 0], [4 + ln2, 2 + ln2 / 2, 2 * ln2])
    # a reset drops whatever the state holds
    y, h = seq.scan(x, np.zeros((1, 3, 1)), np.array([[-1.0]]), ones, ones, reset=np.array([[1, 0, 0]]),
                    state=np.full((1, 1, 1), np.nan))
    assert np.isfinite(y).all() and np.isfinite(h).all()


def scan_inputs(r, batch, time, ch, n, groups):
    return dict(x=r.standard_normal((batch, time, ch)), dt=0.5 * r.standard_normal((batch, time, ch)),
                a=-np.exp(r.standard_normal((ch, n))), b=r.standard_normal((batch, time, groups * n)),
                c=r.standard_normal((batch, time, groups * n)), d=r.standard_normal(ch),
                z=r.standard_normal((batch, time, ch)), dt_bias=r.standard_normal(ch),
                state=r.standard_normal((batch, ch, n)))


@pytest.mark.parametrize("groups", [1, 2])
def test_scan_gradient_against_differences(groups):
    r = rng(5)
    k = scan_inputs(r, 2, 6, 4, 3, groups)
    reset = np.zeros((2, 6), dtype=np.uint8)
    reset[1, 3] = 1
    dy, dh = r.standard_normal((2, 6, 4)), r.standard_normal((2, 4, 3))
    grads = seq.scan_grad(dy, reset=reset, dstate_out=dh, groups=groups, **k)

    def loss(kk):
        y, h = seq.scan(reset=reset, groups=groups, **kk)
        return (y * dy).sum() + (h * dh).sum()

    for name in k:
        v = r.standard_normal(k[name].shape)
        eps = 1e-5
        diff = (loss({**k, name: k[name] + eps * v}) - loss({**k, name: k[name] - eps * v})) / (2 * eps)
        got = (grads["d" + name] * v).sum()
        assert abs(diff - got) < 1e-6 * (1 + abs(got)), name


def test_conv_gradient_against_differences():
    r = rng(6)
    k = dict(x=r.standard_normal((2, 7, 3)), w=r.standard_normal((3, 4)), bias=r.standard_normal(3))
    history, reset = r.standard_normal((2, 3, 3)), np.zeros((2, 7), dtype=np.uint8)
    reset[0, 2] = reset[0, 3] = reset[1, 0] = 1
    dy = r.standard_normal((2, 7, 3))
    dx, dw, dbias = seq.conv_grad(dy, reset=reset, history=history, **k)
    for name, grad in (("x", dx), ("w", dw), ("bias", dbias)):
        v = r.standard_normal(k[name].shape)
        eps = 1e-5
        hi = (seq.conv(reset=reset, history=history, **{**k, name: k[name] + eps * v})[0] * dy).sum()
        lo = (seq.conv(reset=reset, history=history, **{**k, name: k[name] - eps * v})[0] * dy).sum()
        assert abs((hi - lo) / (2 * eps) - (grad * v).sum()) < 1e-6 * (1 + abs((grad * v).sum())), name


def test_gated_ffn_gradient_against_differences():
    r = rng(7)
    for act in seq.ACTIVATIONS:
        k = [r.standard_normal((5, 6)), r.standard_normal((8, 6)), r.standard_normal((6, 4))]
        dy = r.standard_normal((5, 6))
        grads = seq.gated_ffn_grad(dy, *k, activation=act)
        for i in range(3):
            v = r.standard_normal(k[i].shape)
            eps = 1e-5
            up, down = list(k), list(k)
            up[i], down[i] = k[i] + eps * v, k[i] - eps * v
            diff = ((seq.gated_ffn(*up, activation=act)[0] - seq.gated_ffn(*down, activation=act)[0]) * dy).sum() / (2 * eps)
            assert abs(diff - (grads[i] * v).sum()) < 1e-6 * (1 + abs((grads[i] * v).sum()))


def test_cutting_a_sequence_changes_nothing():
    r = rng(8)
    k = scan_inputs(r, 3, 9, 4, 5, 1)
    reset = (r.random((3, 9)) < 0.3).astype(np.uint8)
    y, h = seq.scan(reset=reset, **k)
    cut = 4
    head = {n: (v[:, :cut] if n in ("x", "dt", "b", "c", "z") else v) for n, v in k.items()}
    tail = {n: (v[:, cut:] if n in ("x", "dt", "b", "c", "z") else v) for n, v in k.items()}
    y0, h0 = seq.scan(reset=reset[:, :cut], **head)
    tail["state"] = h0
    y1, h1 = seq.scan(reset=reset[:, cut:], **tail)
    assert np.allclose(np.concatenate([y0, y1], axis=1), y) and np.allclose(h1, h)
    x, w, bias = k["x"], r.standard_normal((4, 3)), r.standard_normal(4)
    y, hist = seq.conv(x, w, bias, reset)
    pieces, carry = [], None
    for t in range(9):
        p, carry = seq.conv(x[:, t:t + 1], w, bias, reset[:, t:t + 1], carry)
        pieces.append(p)
    assert np.allclose(np.concatenate(pieces, axis=1), y) and np.allclose(carry, hist)
