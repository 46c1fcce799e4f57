"""The scan and the convolution over the loops that large calls run in: many steps, several chunks per
segment, several rows per block, whole vectors.  Cases state how their work is cut and check it, so that a
change of the cut cannot leave a loop without a test.
"""
import numpy as np
import pytest

from oracle import sequence as seq
from paper_2603_12145_b200 import ssm

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -23


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
