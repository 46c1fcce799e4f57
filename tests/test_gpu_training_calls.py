"""Calls of the training operators (layer norm, gated recurrence, orthogonalised update) that their own files leave out."""
import numpy as np
import pytest

from oracle import training as tr
from paper_2603_12145_b200 import gated_recurrence, layer_norm, optimizers, orthogonal, ssm_policy
from test_gpu_gated_recurrence import bounds, make, near
from test_gpu_layer_norm import check_backward, check_forward
from test_gpu_layer_norm import make as rows_of
from test_gpu_orthogonal import BOUND, error, matrices

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
    the gate itself times x = 1.  In units of 2^-24 a sigmoid has at most 12 (four of the exponential, 115 * 2e-9 / 2^-24 = 4 of its
    exponent, one of 1 + e, two of the reciprocal, one of a product), the products and the last rounding one each: 16; its derivative a
    sigmoid and the exponential more: 32.  The exponent rounded to one number would be off by 62 at -80."""
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


def roundings_of_da(op, batch, time, ch, cut):
    """Roundings that a term of da passes: of its four steps, the tiles of its slot one after the other, the slots by eights, these
    eight.  The slots from the backward workspace, [slots][channels] behind two states per piece where the time is cut (each then
    a slot of its own)."""
    rows = op._size(batch, time, 1) // (4 * ch)
    slots = rows // 3 if cut else rows
    assert slots >= batch if cut else slots <= batch
    tiles = -(-batch // slots) * -(-time // 4) if not cut else -(-time * batch // (4 * slots)) + 2
    return 4 + tiles + slots / 8 + 9


@pytest.mark.parametrize("case", [(2500, 19, 70, "float32", False), (300, 40, 257, "bfloat16", False), (1, 16000, 64, "bfloat16", True),
                                  (3, 777, 40, "float16", True)], ids=str)
def test_the_rates_gradient_to_the_roundings_of_its_own_sum(torch, case):
    """da within what the sum's own chains may cost, some ten to a hundred roundings."""
    batch, time, ch, dtype, cut = case
    dev, val = make(torch, 40 + time, batch, time, ch, dtype, "batch", 0.0, True)
    op = gated_recurrence.GatedRecurrence(ch, dtype=getattr(torch, dtype))
    four = [dev[k] for k in ("x", "r", "i", "a")]
    saved = op.saved(batch, time)
    op.sequence(*four, state=dev["state"], saved=saved)
    g = op.backward(dev["dy"], *four, saved, dstate_out=dev["dstate_out"])
    want = tr.recurrence_grad(val["dy"], *(val[k] for k in ("x", "r", "i", "a")), None, val["state"], val["dstate_out"])["da"]
    units, sums = bounds(val)
    near("da", g["da"], want, units["da"] + roundings_of_da(op, batch, time, ch, cut) * sums)


@pytest.mark.parametrize("batch,time,ch,rows", [(1, 2000, 2000, 1), (1, 1, 33, 1), (2, 1003, 1000, 2), (1300, 19, 1140, 60), (900, 40, 800, 20)])
def test_every_step_counts_once_in_the_rates_gradient(torch, batch, time, ch, rows):
    """One gradient per channel, each at another row and step, in channels that forget at once: da is then a few terms, and one that
    is left out or taken twice is most of it.  All steps of one row, of two; rows from the first, the middle and the last ones (several
    share a slot), at every step.  The few terms add up within eight roundings beyond the operator's bounds."""
    r = np.random.Generator(np.random.PCG64(time))
    op = gated_recurrence.GatedRecurrence(ch, dtype=torch.float32)
    for turn in range(max(1, -(-rows * time // ch))):
        pos = (np.arange(ch) + turn * ch) % (rows * time)
        row, step = pos // time, pos % time
        row = np.where(row % 3 == 0, row, np.where(row % 3 == 1, batch - 1 - row, batch // 2 + row)) if rows > 2 else row
        val = {k: r.standard_normal((batch, time, ch)).astype(np.float32) for k in ("x", "r", "i")}
        val["a"] = -np.exp(r.uniform(np.log(1.0), np.log(8.0), ch)).astype(np.float32)
        val["dy"] = np.zeros((batch, time, ch), np.float32)
        val["dy"][row, step, np.arange(ch)] = 1.0
        val.update(state=r.standard_normal((batch, ch)).astype(np.float32), dstate_out=None, reset=None)
        dev = {k: None if v is None else torch.from_numpy(v).cuda() for k, v in val.items()}
        four = [dev[k] for k in ("x", "r", "i", "a")]
        saved = op.saved(batch, time)
        op.sequence(*four, state=dev["state"], saved=saved)
        g = op.backward(dev["dy"], *four, saved)
        # the definition on the rows that have one, those before the step only by what is left of them
        used = np.unique(row)
        small = {k: (v if v is None or k == "a" else np.asarray(v, np.float64)[used]) for k, v in val.items()}
        want = tr.recurrence_grad(small["dy"], *(small[k] for k in ("x", "r", "i", "a")), None, small["state"])["da"]
        units, sums = bounds(small)
        near("da", g["da"], want, units["da"] + 8 * sums)
        assert (np.abs(want) > 100 * (units["da"] + 8 * sums) * U).mean() > 0.9       # a lost term would be seen


# ---- layer norm -------------------------------------------------------------------------


@pytest.mark.parametrize("width,dtype", [(577, "bfloat16"), (577, "float16"), (1501, "bfloat16"), (301, "float16"), (2903, "bfloat16")])
def test_in_place_between_boundaries(torch, width, dtype):
    """Rows whose accesses reach into their neighbours, which others are writing at the same time."""
    n, t = 4001, getattr(torch, dtype)
    op = layer_norm.LayerNorm(width, dtype=t)
    x, r, dy, d = (normal(torch, k, n, width, dtype=t) for k in range(4))
    w, b = normal(torch, 5, width), normal(torch, 6, width)
    saved = op.saved(n)
    y, s = op.forward(x, w, b, residual=r, saved=saved)
    plain = op.forward(s, w, b)
    want = op.backward(dy, s, w, saved, dsum=d)
    for _ in range(3):
        x2, r2, z, again = x.clone(), r.clone(), s.clone(), op.saved(n)
        y2, s2 = op.forward(x2, w, b, residual=r, total=x2, saved=again)
        assert s2 is x2 and torch.equal(x2, s) and torch.equal(y2, y) and torch.equal(again, saved)
        y3, s3 = op.forward(x, w, b, residual=r2, total=r2)
        assert s3 is r2 and torch.equal(r2, s) and torch.equal(y3, y)
        assert torch.equal(op.forward(z, w, b, out=z), plain)
        for k in range(2):
            dy2, d2 = dy.clone(), d.clone()
            got = op.backward(dy2, s, w, saved, dsum=d2, out=(dy2, d2)[k])
            assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("width", [64, 577, 1501, 2048, 4001])
def test_nan_and_infinity_stay_in_their_rows_backward(torch, width):
    n, t = 700, torch.bfloat16
    op = layer_norm.LayerNorm(width, dtype=t)
    s, dy, d = (normal(torch, k, n, width, dtype=t) for k in range(3))
    saved = op.saved(n)
    op.forward(s, saved=saved)
    clean = op.backward(dy, s, None, saved, dsum=d)[0]
    for which in range(3):
        bad = [v.clone() for v in (s, dy, d)]
        bad[which][3, width // 2] = float("nan")
        bad[which][11, 0] = float("inf")
        bad[which][n - 1, width - 1] = float("-inf")
        kept = op.saved(n)
        op.forward(bad[0], saved=kept)
        dx = op.backward(bad[1], bad[0], None, kept, dsum=bad[2])[0]
        hit = torch.zeros((n, width), dtype=torch.bool, device="cuda")
        hit[[3, 11, n - 1]] = True
        if which == 2:                       # it is added at the end: the element alone
            hit = ~torch.isfinite(bad[2])
        assert not torch.isfinite(dx[hit]).any() and torch.equal(dx[~hit], clean[~hit])


@pytest.mark.parametrize("n,width,dtype", [(300, 576, "bfloat16"), (300, 1024, "float16"), (300, 512, "float32"), (9, 8192, "bfloat16"), (40, 72, "bfloat16")])
def test_parameters_off_boundaries(torch, n, width, dtype):
    """Whole rows, weights that begin one element behind a boundary of 16 bytes."""
    op = layer_norm.LayerNorm(width, eps=1e-5, dtype=getattr(torch, dtype))
    x, r, dy, d = (rows_of(torch, k, n, width, dtype) for k in range(1, 5))
    w, b = (normal(torch, k, width + 1)[1:] for k in (5, 6))
    assert w.data_ptr() % 16 == 4
    saved = op.saved(n)
    y, s = op.forward(x, w, b, residual=r, saved=saved)
    assert torch.equal(s, x + r)
    check_forward(f64(s), y, f64(w), f64(b), 1e-5, dtype)
    dx, dw, db = op.backward(dy, s, w, saved, dsum=d)
    check_backward(f64(s), f64(dy), f64(w), f64(d), 1e-5, dtype, dx, dw, db)


# ---- orthogonalised update ----------------------------------------------------------------

# Sizes that go between all blocks: either way round, rows of G and of the update on boundaries and off them.
LARGE = [(200, 304), (304, 200), (197, 333), (333, 197), (640, 1024)]


@pytest.mark.parametrize("rows,cols", LARGE)
def test_large_nan_stays_in_its_matrix(torch, rows, cols):
    g = matrices(torch, 6, 4, rows, cols, "bfloat16")
    op = orthogonal.Orthogonal(rows, cols)
    clean = op.update(g)
    g[1, rows - 1, 3] = float("nan")
    g[3, 0, cols - 1] = float("inf")
    out = op.update(g)
    op.status()
    assert torch.isnan(out[1]).all() and torch.isnan(out[3]).all()
    assert torch.equal(out[0], clean[0]) and torch.equal(out[2], clean[2])


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows,cols", LARGE)
def test_large_strides_and_surroundings(torch, rows, cols, dtype):
    """G in columns of a wider array, transposed batches, one matrix for all; the update into a part of an array, on and off
    boundaries of 16 bytes."""
    op = orthogonal.Orthogonal(rows, cols, dtype=getattr(torch, dtype))
    g = matrices(torch, 7, 3, rows, cols, dtype)
    want = op.update(g)
    for z in range(3):
        assert error(want[z], tr.orthogonal(f64(g[z]))) <= BOUND
    for pad, at in ((9, 5), (16, 8)):
        wide = torch.full((3, rows, cols + pad), float("nan"), dtype=g.dtype, device="cuda")
        wide[:, :, at:at + cols] = g
        assert torch.equal(op.update(wide[:, :, at:at + cols]), want)
        big = torch.full((3, rows + 2, cols + pad), 7.0, dtype=torch.bfloat16, device="cuda")
        op.update(g, out=big[:, 1:1 + rows, at:at + cols])
        assert torch.equal(big[:, 1:1 + rows, at:at + cols], want)
        big[:, 1:1 + rows, at:at + cols] = 7.0
        assert (big == 7.0).all()
    inner = g.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(op.update(inner), want)
    assert torch.equal(op.update(g[1:2].expand(3, rows, cols)), want[1:2].expand(3, rows, cols))
    op.status()


@pytest.mark.parametrize("nesterov,decay", [(True, 0.0), (False, 0.1)])
def test_orthogonal_momentum_takes_its_steps(torch, nesterov, decay):
    """Three steps on matrices of both forms, two of one shape, against the formula in binary64 with the oracle's products.  A
    step's update is off by at most BOUND of its norm; the weights' roundings are 3 * 3 * 2^-24 of at most 4 each."""
    shapes = [(96, 40), (96, 40), (200, 304), (500, 300)]
    params = [torch.nn.Parameter(0.1 * normal(torch, k, *s)) for k, s in enumerate(shapes)]
    opt = optimizers.OrthogonalMomentum(params, lr=0.02, momentum=0.9, nesterov=nesterov, weight_decay=decay)
    want, m, room = [f64(p.detach()) for p in params], [0.0] * 4, [0.0] * 4
    for step in range(3):
        for k, (rows, cols) in enumerate(shapes):
            params[k].grad = matrices(torch, 10 * step + k, 1, rows, cols, "float32", 4, 0.3)[0]
            g = f64(params[k].grad)
            m[k] = 0.9 * m[k] + g
            update = 0.02 * max(1.0, rows / cols) ** 0.5 * tr.orthogonal(g + 0.9 * m[k] if nesterov else m[k])
            want[k] = (1.0 - 0.02 * decay) * want[k] - update
            room[k] += BOUND * np.linalg.norm(update) + 9 * U * 4 * (rows * cols) ** 0.5
        opt.step()
    opt.check()
    for k, p in enumerate(params):
        assert np.linalg.norm(f64(p.detach()) - want[k]) <= room[k], k


# ---- the policy without the new choices ------------------------------------------------------


def test_the_default_policy_computes_what_it_did(torch):
    """Its layer written out as it was before it had a choice of mixer and norm, from the same operators: the same bits, of the
    logits in one piece and by single tokens, of the carried state and of every gradient."""
    policy = ssm_policy.StateSpacePolicy(model=64, layers=2, ffn_hidden=72)
    conv, scan, ffn = ssm_policy.ConvFunction.apply, ssm_policy.ScanFunction.apply, ssm_policy.FfnFunction.apply
    batch, time = 5, 20
    obs = normal(torch, 1, batch, time, 6)
    reset = (torch.rand((batch, time), generator=torch.Generator("cuda").manual_seed(2), device="cuda") < 0.1).to(torch.uint8)
    done = reset.t().contiguous()
    carry = [(normal(torch, 3, *s.shape), normal(torch, 4, *h.shape, dtype=h.dtype)) for s, h in policy.start(batch)]

    def sequence():
        h = (obs @ policy.embed.t()).to(torch.bfloat16)
        for layer, (state, history) in zip(policy.layers, carry):
            x, z = torch.split(h @ layer.w_xz.to(h.dtype).t(), [layer.inner, layer.inner], dim=-1)
            x = conv(layer.op, x, layer.conv_w, layer.conv_b, reset, history, None)
            r, b, c = torch.split(x @ layer.w_p.to(x.dtype).t(), [layer.rank, layer.states, layer.states], dim=-1)
            y = scan(layer.op, x, r @ layer.w_dt.to(x.dtype).t(), -torch.exp(layer.log_rate), b, c, layer.skip, z, layer.dt_bias, reset,
                     state, None)
            h = h + y @ layer.w_y.to(h.dtype).t()
            rows = h.transpose(0, 1).reshape(batch * time, 64)
            f = ffn(layer.ffn, rows, layer.w_in.to(h.dtype), layer.w_out.to(h.dtype))
            h = h + f.view(time, batch, 64).transpose(0, 1)
        return h.float() @ policy.head.t()

    def step(t, carry):
        h = (obs[:, t] @ policy.embed.t()).to(torch.bfloat16)
        for layer, (state, history) in zip(policy.layers, carry):
            w = {k: getattr(layer, k).detach().to(torch.bfloat16) for k in ("w_xz", "w_p", "w_dt", "w_y", "w_in", "w_out")}
            x, z = torch.split(h @ w["w_xz"].t(), [layer.inner, layer.inner], dim=-1)
            x = layer.op.conv_step(x, history, layer.conv_w, layer.conv_b, done=done[t])
            r, b, c = torch.split(x @ w["w_p"].t(), [layer.rank, layer.states, layer.states], dim=-1)
            y = layer.op.scan_step(x, r @ w["w_dt"].t(), -torch.exp(layer.log_rate.detach()), b, c, state, d=layer.skip, z=z,
                                   dt_bias=layer.dt_bias, done=done[t])
            h = h + y @ w["w_y"].t()
            h = h + layer.ffn.forward(h, w["w_in"], w["w_out"])
        return h.float() @ policy.head.t()

    k = normal(torch, 9, batch, time, 3)
    names, params = zip(*policy.named_parameters())
    a, b = policy.sequence(obs, reset, carry), sequence()
    assert torch.equal(a, b)
    for name, p, q in zip(names, torch.autograd.grad((a * k).sum(), params), torch.autograd.grad((b * k).sum(), params)):
        assert torch.equal(p, q), name
    one, two = ([(s.clone(), h.clone()) for s, h in carry] for _ in range(2))
    weights = policy.weights()
    with torch.no_grad():
        for t in range(4):
            assert torch.equal(policy.step(obs[:, t], done[t], one, weights), step(t, two))
    assert all(torch.equal(p, q) for u, v in zip(one, two) for p, q in zip(u, v))
    for layer in policy.layers:
        layer.ffn.status()
