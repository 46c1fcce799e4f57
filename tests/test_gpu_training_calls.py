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
