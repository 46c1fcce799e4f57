"""The binary64 definitions of oracle/training.py: hand-computed cases, central differences, invariances."""
import numpy as np
import pytest

from oracle import training as tr


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def central(f, v, d, h=1e-6):
    """sum(d * f(v)) differentiated along every element of v."""
    out = np.empty_like(v)
    for k in np.ndindex(v.shape):
        up, down = v.copy(), v.copy()
        up[k] += h
        down[k] -= h
        out[k] = ((d * f(up)).sum() - (d * f(down)).sum()) / (2 * h)
    return out


def test_norm_by_hand():
    y, mean, scale = tr.norm([[1.0, 3.0], [5.0, 5.0]], w=[2.0, 1.0], b=[0.5, 0.0], eps=3.0)
    assert np.allclose(mean, [2.0, 5.0]) and np.allclose(scale, [0.5, 1 / np.sqrt(3.0)])
    assert np.allclose(y, [[-0.5, 0.5], [0.5, 0.0]])


def test_norm_gradients_against_differences():
    r = rng(1)
    s, w, b, dy = r.standard_normal((3, 7)), r.standard_normal(7), r.standard_normal(7), r.standard_normal((3, 7))
    dx, dw, db = tr.norm_grad(dy, s, w)
    assert np.allclose(dx, central(lambda v: tr.norm(v, w, b)[0], s, dy), atol=1e-7)
    assert np.allclose(dw, central(lambda v: tr.norm(s, v, b)[0], w, dy), atol=1e-7)
    assert np.allclose(db, central(lambda v: tr.norm(s, w, v)[0], b, dy), atol=1e-7)
    assert np.allclose(tr.norm_grad(dy, s, w, dsum=s)[0], dx + s)


def test_recurrence_by_hand():
    # sigmoid(0) = 1/2: decay e^(a/2), here 1/2, so the gain is sqrt(3)/2
    a = np.array([2.0 * np.log(0.5)])
    x = np.array([[[4.0], [8.0]]])
    zero = np.zeros_like(x)
    y, last, before = tr.recurrence(x, zero, zero, a, state=np.array([[6.0]]))
    k = np.sqrt(0.75)
    assert np.allclose(y[0, :, 0], [3.0 + 2.0 * k, 1.5 + k + 4.0 * k]) and np.allclose(last, y[:, 1])
    assert np.allclose(before[0, :, 0], [6.0, 3.0 + 2.0 * k])
    y, _, before = tr.recurrence(x, zero, zero, a, reset=np.array([[0, 1]]), state=np.array([[np.inf]]))
    assert np.isinf(y[0, 0, 0]) and np.isclose(y[0, 1, 0], 4.0 * k) and before[0, 1, 0] == 0.0


@pytest.mark.parametrize("reset", [None, np.array([[0, 1, 0, 0, 1], [1, 0, 0, 0, 0]])])
def test_recurrence_gradients_against_differences(reset):
    r = rng(2)
    x, g, i, dy = (r.standard_normal((2, 5, 3)) for _ in range(4))
    a, state, dlast = -np.exp(r.standard_normal(3)), r.standard_normal((2, 3)), r.standard_normal((2, 3))

    def both(**change):
        args = dict(x=x, r=g, i=i, a=a, state=state)
        args.update(change)
        y, last, _ = tr.recurrence(reset=reset, **args)
        return np.concatenate([y.ravel(), last.ravel()])

    d = np.concatenate([dy.ravel(), dlast.ravel()])
    got = tr.recurrence_grad(dy, x, g, i, a, reset, state, dlast)
    for key, name, v in (("dx", "x", x), ("dr", "r", g), ("di", "i", i), ("da", "a", a), ("dstate", "state", state)):
        assert np.allclose(got[key], central(lambda u: both(**{name: u}), v, d), atol=1e-6), key
    mag = tr.recurrence_grad(dy, x, g, i, a, reset, state, dlast, magnitude=True)
    assert all((mag[k] >= np.abs(got[k]) - 1e-12).all() for k in got)


def test_recurrence_in_two_pieces_is_the_recurrence():
    r = rng(3)
    x, g, i = (r.standard_normal((2, 9, 4)) for _ in range(3))
    a, state = -np.exp(r.standard_normal(4)), r.standard_normal((2, 4))
    whole = tr.recurrence(x, g, i, a, state=state)
    first = tr.recurrence(x[:, :4], g[:, :4], i[:, :4], a, state=state)
    second = tr.recurrence(x[:, 4:], g[:, 4:], i[:, 4:], a, state=first[1])
    assert np.allclose(np.concatenate([first[0], second[0]], axis=1), whole[0]) and np.allclose(second[1], whole[1])


def test_recurrence_keeps_the_variance_of_white_inputs():
    """The gain sqrt(1 - decay^2) makes a unit-variance input's state one of unit variance."""
    r = rng(4)
    x = r.standard_normal((400, 200, 1))
    big = np.full_like(x, 50.0)
    y, _, _ = tr.recurrence(x, big, big, np.array([-0.05]))
    assert abs(y[:, -50:].var() - 1.0) < 0.1


def test_orthogonal_is_the_polynomial_of_the_singular_values():
    r = rng(5)
    a, b, c = tr.COEFFICIENTS
    for shape in ((5, 9), (9, 5), (6, 6), (1, 4)):
        g = r.standard_normal(shape)
        u, s, vt = np.linalg.svd(g, full_matrices=False)
        s = s / (np.sqrt((s * s).sum()) + 1e-7)
        for _ in range(5):
            s = a * s + b * s ** 3 + c * s ** 5
        assert np.allclose(tr.orthogonal(g), (u * s) @ vt)
        assert np.allclose(tr.orthogonal(g.T), tr.orthogonal(g).T)
    assert (tr.orthogonal(np.zeros((3, 4))) == 0.0).all()
    assert 0.6 < np.abs(tr.orthogonal(np.array([[-7.0]]))).item() < 1.3
