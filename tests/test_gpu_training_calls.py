"""Calls of the training operators (layer norm, gated recurrence, orthogonalised update) that their own files leave out."""
import numpy as np
import pytest

from oracle import training as tr
from paper_2603_12145_b200 import gated_recurrence, ssm_policy

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    from paper_2603_12145_b200 import build
    assert torch.cuda.is_available()
    build.build()
    return torch


def f64(t):
    return t.double().cpu().numpy()


def normal(torch, seed, *shape, dtype=None):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype or torch.float32)


# ---- gated recurrence -----------------------------------------------------------------


@pytest.mark.parametrize("batch,time,reset", [(7, 1, 0.0), (5, 24, 0.2), (1, 700, 0.0)])
def test_the_state_at_the_start_has_its_gradient(torch, batch, time, reset):
    """Through autograd, against the formula in binary64.  A term that comes back over n steps has a relative error of at most
    (64 S + 2 n + 64) 2^-24, S the sum of their 1 - e^L (a step's own bound, test_gpu_gated_recurrence.py), and weighs e^-S: beyond
    S = 32 nothing is left of it, so that with n <= 700 the error is below 2^-12 of the terms' magnitudes."""
    ch = 40
    x, r, i = (normal(torch, 30 + k, batch, time, ch) for k in range(3))
    a = -torch.exp(normal(torch, 34, ch).abs()) / 20
    dy = normal(torch, 35, batch, time, ch)
    mask = (torch.rand((batch, time), generator=torch.Generator("cuda").manual_seed(36), device="cuda") < reset).to(torch.uint8)
    state = normal(torch, 37, batch, ch).requires_grad_(True)
    op = gated_recurrence.GatedRecurrence(ch, dtype=torch.float32)
    y = ssm_policy.RecurrenceFunction.apply(op, x, r, i, a, mask, state, None)
    (got,) = torch.autograd.grad((y * dy).sum(), state)
    v = [f64(t) for t in (dy, x, r, i, a)]
    want = tr.recurrence_grad(*v, mask.cpu().numpy(), f64(state.detach()))["dstate"]
    size = tr.recurrence_grad(*v, mask.cpu().numpy(), f64(state.detach()), magnitude=True)["dstate"]
    assert (np.abs(f64(got) - want) <= 2.0 ** -12 * size).all()
    assert np.abs(want).max() > 0.1


def test_overlapping_windows_as_input(torch):
    """x, r and i as windows into a series, a step or a row apart: what dense copies give."""
    batch, time, ch = 6, 30, 24
    op = gated_recurrence.GatedRecurrence(ch, dtype=torch.float32)
    a, dy = -torch.exp(normal(torch, 1, ch)), normal(torch, 2, batch, time, ch)
    for strides in ((time, 1, 1), (1, batch, 1), (1, 1, 1), (0, ch, 1), (0, 0, 1)):
        x, r, i = (normal(torch, 3 + k, 1000).as_strided((batch, time, ch), strides) for k in range(3))
        dense = [v.contiguous() for v in (x, r, i)]
        saved, kept = op.saved(batch, time), op.saved(batch, time)
        assert torch.equal(op.sequence(x, r, i, a, saved=saved), op.sequence(*dense, a, saved=kept))
        got, want = op.backward(dy, x, r, i, a, saved), op.backward(dy, *dense, a, kept)
        assert all(torch.equal(got[k], want[k]) for k in ("dx", "dr", "di", "da"))


@pytest.mark.parametrize("ch", [64, 33])
def test_binary32_gates_keep_their_relative_precision(torch, ch):
    """Input gates from all but closed (e^-80) to all but open, with a decay that is nothing (a = -50, its gate open), so that y is
    the gate itself times x = 1.  In units of 2^-24 a sigmoid has 8 (four of the exponential, one of 1 + e, two of the reciprocal,
    one of the exponent's low part), the gain's root 4, the products and the last rounding one each: 16; its derivative a sigmoid
    and the exponential more: 32.  The exponent rounded to one number would be off by 62 at -80."""
    n = 2000
    op = gated_recurrence.GatedRecurrence(ch, dtype=torch.float32)
    gate = torch.linspace(-80.0, 80.0, n * ch, device="cuda").view(n, 1, ch)
    x, r, a = torch.ones_like(gate), torch.full_like(gate, 60.0), torch.full((ch,), -50.0, device="cuda")
    si = tr.sigmoid(f64(gate))
    saved = op.saved(n, 1)
    got = op.sequence(x, r, gate, a, saved=saved)
    g = op.backward(x, x, r, gate, a, saved)
    one = op.step(x[:, 0], r[:, 0], gate[:, 0], a, torch.zeros((n, ch), device="cuda"))
    slope = si * tr.sigmoid(-f64(gate))
    for name, v, want, units in (("y", got, si, 16), ("step", one[:, None], si, 16), ("dx", g["dx"], si, 16), ("di", g["di"], slope, 32)):
        err = np.abs(f64(v) / want - 1.0).max() / U
        assert err <= units, (name, err)


def test_binary32_gates_of_any_size(torch):
    """Infinite, huge and vanishing gates, and one that is no number, in its channel alone."""
    v = torch.tensor([float("-inf"), -3e38, -104.0, -88.5, -87.4, 0.0, 90.0, 3e38, float("inf"), float("nan")], device="cuda")
    op = gated_recurrence.GatedRecurrence(10, dtype=torch.float32)
    x, a = torch.ones((3, 5, 10), device="cuda"), torch.full((10,), -1.0, device="cuda")
    open_ = torch.full_like(x, 60.0)
    gate = v.expand(3, 5, 10).contiguous()
    for r, i in ((open_, gate), (gate, open_)):
        saved = op.saved(3, 5)
        y = op.sequence(x, r, i, a, state=torch.ones((3, 10), device="cuda"), saved=saved)
        g = op.backward(x, x, r, i, a, saved)
        for out in (y, g["dx"], g["dr"], g["di"]):
            assert torch.isfinite(out[..., :9]).all() and torch.isnan(out[..., 9]).all()
