"""The gated feed-forward block against the binary64 oracle, through the binding.

Tolerances, with u the type's unit roundoff (2^-8 bfloat16, 2^-11 binary16) and 2^-23 per addition
of a binary32 accumulation over K terms (the order is unspecified; each step loses at most
that much of the running sum, which the sum S of absolute terms bounds).  Forward:

    g, u        |error| <= K 2^-23 S_in                                           =: e_in
    hidden      |error| <= u |hidden| + 1.2 (|u| + |act(g)| + 1) e_in + 2^-21 |hidden|    =: e_h
    y           |error| <= u |y| + e_h |W_out|^T + K 2^-23 |hidden| |W_out|^T

(|act'| <= 1.13 for both activations; a few units of binary32 for exponential and reciprocal).
Backward, from the pre-activations rounded to the type (g moves by u |g|: act' changes by at most
1.1 u |g| and act by 1.13 u |g|):

    dhidden     |error| <= K 2^-23 |dy| |W_out|
    dg          |error| <= u |dg| + 1.13 |u_pre| e_dh + |dhidden| (1.13 u |u_pre| + |u_pre| 1.1 u |g|)
    du          |error| <= u |du| + 1.2 |g| e_dh + |dhidden| 1.2 u (|g| + 1)
    products    the operands' errors times the other operand's absolute values, plus K 2^-23 S, plus u |result|

with a tenth added for second-order terms.  Results below the least normal binary16 number may be
off by its spacing.
"""
import numpy as np
import pytest

from oracle import sequence as seq
from paper_2603_12145_b200 import gated_ffn as gf

pytestmark = pytest.mark.gpu

UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
EPS = 2.0 ** -23


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    gf.load(build_if_missing=True)
    return torch


def device(torch, a, dtype, pad=0):
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda().to(getattr(torch, dtype))
    values = t.double().cpu().numpy()
    if pad:
        wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
        wide[:, :t.shape[1]] = t
        t = wide[:, :t.shape[1]]
    return t, values


def check(name, got, want, tol, dtype):
    got = got.double().cpu().numpy()
    tol = 1.1 * tol + UNIT[dtype] * np.abs(want) + (2.0 ** -24 if dtype == "float16" else 0.0)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, first at %s: got %r want %r tol %r" % (
        name, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])


def bounds(x, w_in, w_out, dy, activation, dtype):
    """The error bounds of the docstring: y, dx, dw_in, dw_out."""
    u, f = UNIT[dtype], w_out.shape[1]
    act, slope = seq.ACTIVATIONS[activation]
    _, pre, hidden = seq.gated_ffn(x, w_in, w_out, activation)
    g, up = pre[:, :f], pre[:, f:]
    e_in = w_in.shape[1] * EPS * (np.abs(x) @ np.abs(w_in).T)
    least = 2.0 ** -24 if dtype == "float16" else 0.0      # spacing of the subnormal numbers
    e_h = u * np.abs(hidden) + 1.2 * (np.abs(up) * e_in[:, :f] + np.abs(act(g)) * e_in[:, f:]
                                     + e_in[:, :f] * e_in[:, f:]) + 2.0 ** -21 * np.abs(hidden) + least
    wo = np.abs(w_out)
    out = {"y": e_h @ wo.T + f * EPS * (np.abs(hidden) @ wo.T)}
    if dy is None:
        return out
    dh = dy @ w_out
    e_dh = w_out.shape[0] * EPS * (np.abs(dy) @ wo)
    # pre as stored: rounded to the type, after the accumulation error
    e_g, e_u = u * np.abs(g) + e_in[:, :f] + least, u * np.abs(up) + e_in[:, f:] + least
    dg, du = dh * up * slope(g), dh * act(g)
    e_dg = u * np.abs(dg) + 1.13 * np.abs(up) * e_dh + np.abs(dh) * (1.13 * e_u + 1.1 * np.abs(up) * e_g) + 2.0 ** -21 * np.abs(dh * up) + least
    e_du = u * np.abs(du) + np.abs(act(g)) * e_dh + np.abs(dh) * 1.13 * e_g + 2.0 ** -21 * np.abs(du) + least
    dpre, e_dpre = np.abs(np.concatenate([dg, du], 1)), np.concatenate([e_dg, e_du], 1)
    n = x.shape[0]
    out["dx"] = e_dpre @ np.abs(w_in) + 2 * f * EPS * (dpre @ np.abs(w_in))
    out["dw_in"] = e_dpre.T @ np.abs(x) + n * EPS * (dpre.T @ np.abs(x))
    out["dw_out"] = np.abs(dy).T @ e_h + n * EPS * (np.abs(dy).T @ np.abs(hidden))
    return out


CASES = [
    # rows, model, hidden, activation, dtype, padding of the rows
    (1, 8, 8, "silu", "bfloat16", 0), (1, 200, 136, "gelu", "float16", 8), (5, 72, 40, "silu", "float16", 0),
    (8, 256, 128, "silu", "bfloat16", 0), (17, 136, 264, "gelu", "bfloat16", 16), (32, 64, 72, "silu", "bfloat16", 8),
    (33, 64, 72, "silu", "bfloat16", 8), (64, 576, 1536, "silu", "bfloat16", 0), (100, 192, 384, "gelu", "float16", 0),
    (255, 128, 320, "silu", "bfloat16", 24), (257, 264, 104, "gelu", "float16", 8), (1003, 328, 520, "silu", "bfloat16", 0),
    (700, 1600, 2304, "gelu", "bfloat16", 0), (3000, 320, 448, "silu", "float16", 0), (129, 2056, 1032, "silu", "float16", 0)]


def operands(seed, n, model, hidden, scale=1.0):
    r = np.random.Generator(np.random.PCG64(seed))
    return (r.standard_normal((n, model)), r.standard_normal((2 * hidden, model)) * scale * model ** -0.5,
            r.standard_normal((model, hidden)) * hidden ** -0.5, r.standard_normal((n, model)))


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward_and_backward(torch, case):
    n, model, hidden, activation, dtype, pad = case
    x, w_in, w_out, dy = operands(n + model, n, model, hidden)
    (xd, x), (wi, w_in), (wo, w_out), (dyd, dy) = (device(torch, x, dtype, pad), device(torch, w_in, dtype),
                                                   device(torch, w_out, dtype), device(torch, dy, dtype, pad))
    want_y, want_pre, want_hidden = seq.gated_ffn(x, w_in, w_out, activation)
    want = dict(zip(("dx", "dw_in", "dw_out"), seq.gated_ffn_grad(dy, x, w_in, w_out, activation)))
    tol = bounds(x, w_in, w_out, dy, activation, dtype)
    op = gf.GatedFfn(model, hidden, activation, getattr(torch, dtype))
    y = op.forward(xd, wi, wo)
    op.status()
    check("y", y, want_y, tol["y"], dtype)
    saved = op.saved(n)
    wide = torch.full((n, model + 8), 7.0, dtype=xd.dtype, device="cuda")
    y2 = op.forward(xd, wi, wo, saved=saved, out=wide[:, :model])
    assert torch.equal(y, y2) and bool((wide[:, model:] == 7.0).all())
    got = dict(zip(("dx", "dw_in", "dw_out"), op.backward(dyd, xd, wi, wo, saved)))
    op.status()
    for key in want:
        check(key, got[key], want[key], tol[key], dtype)
    again = op.backward(dyd, xd, wi, wo, saved, want_dx=False)
    assert again[0] is None and torch.equal(again[1], got["dw_in"]) and torch.equal(again[2], got["dw_out"])
    op.status()


def test_large_products_on_exact_operands(torch):
    """Operands that are small multiples of powers of two make every product and sum exact: the linear
    parts (dw_out from a given hidden, and dx from a given dpre through gate zero) then agree to the
    rounding of the result, at sizes with several rounds of tiles and a divided last one."""
    n, model, hidden = 2500, 1160, 3080
    r = np.random.Generator(np.random.PCG64(5))
    draw = lambda *s: r.integers(-2, 3, s) / 4.0      # noqa: E731
    dy, x, w_in, w_out = draw(n, model), draw(n, model), draw(2 * hidden, model), draw(model, hidden)
    hid, pre = draw(n, hidden), np.concatenate([np.zeros((n, hidden)), draw(n, hidden)], 1)
    dev = [torch.from_numpy(v).cuda().to(torch.bfloat16) for v in (dy, x, w_in, w_out, pre, hid)]
    op = gf.GatedFfn(model, hidden)
    # the pre-activations as the library keeps them: these values fit the upper 16 bits of binary32, so the lower
    # planes are zero
    kept = op.saved(n)[0].zero_()
    kept[:n * 4 * hidden] = dev[4].float().view(torch.int32).bitwise_right_shift(16).to(torch.int16).view(torch.uint8).flatten()
    dx, dw_in, dw_out = op.backward(dev[0], dev[1], dev[2], dev[3], (kept, dev[5]))
    op.status()
    f = [v.double() for v in dev]
    # silu(0) = 0, silu'(0) = 1/2: dg = dhidden up / 2 rounded to the type, du = 0
    dg = (f[0] @ f[3] * f[4][:, hidden:] * 0.5).to(torch.bfloat16).double()
    for got, want, mag in ((dw_out, f[0].t() @ f[5], None), (dx, dg @ f[2][:hidden], dg.abs() @ f[2][:hidden].abs()),
                           (dw_in[:hidden], dg.t() @ f[1], dg.abs().t() @ f[1].abs())):
        tol = 2.0 ** -8 * want.abs() + (0.0 if mag is None else n * EPS * mag)
        assert bool(((got.double() - want).abs() <= tol).all())
    assert bool((dw_in[hidden:] == 0).all())


def test_gradient_against_differences_of_the_kernel(torch):
    """Directional derivatives of the forward kernel (binary16): the loss is a sum over 200 x 64 outputs, each
    with a rounding error of 2^-11 relative; along the gradient, with steps that change the loss by several
    per cent, 3 % is far above both that noise and the third-order term."""
    n, model, hidden = 200, 64, 128
    x, w_in, w_out, dy = operands(3, n, model, hidden)
    dev = [device(torch, v, "float16")[0] for v in (x, w_in, w_out, dy)]
    op = gf.GatedFfn(model, hidden, "gelu", torch.float16)
    saved = op.saved(n)
    op.forward(*dev[:3], saved=saved)
    grads = op.backward(dev[3], *dev[:3], saved)
    for i in range(3):
        v = grads[i].double() / grads[i].double().abs().max()
        eps = 2.0 ** -5
        up, down = list(dev[:3]), list(dev[:3])
        up[i], down[i] = (dev[i].double() + eps * v).half(), (dev[i].double() - eps * v).half()
        moved = up[i].double() - down[i].double()
        diff = ((op.forward(*up).double() - op.forward(*down).double()) * dev[3].double()).sum().item()
        want = (grads[i].double() * moved).sum().item()
        assert abs(diff - want) <= 0.03 * abs(want), (i, diff, want)


def test_a_row_with_nan_stays_alone_and_side_stream(torch):
    n, model, hidden = 300, 128, 256
    x, w_in, w_out, _ = operands(4, n, model, hidden)
    xd, wi, wo = [device(torch, v, "bfloat16")[0] for v in (x, w_in, w_out)]
    op = gf.GatedFfn(model, hidden)
    y = op.forward(xd, wi, wo)
    bad = xd.clone()
    bad[17] = float("nan")
    bad[200, 3] = float("inf")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = op.forward(bad, wi, wo)
    torch.cuda.synchronize()
    keep = [i for i in range(n) if i not in (17, 200)]
    assert torch.equal(z[keep], y[keep]) and bool(torch.isnan(z[17]).all())


def test_refusals(torch):
    op = gf.GatedFfn(64, 128)
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    wi = torch.zeros((256, 64), dtype=torch.bfloat16, device="cuda")
    wo = torch.zeros((64, 128), dtype=torch.bfloat16, device="cuda")
    for bad in ((x.half(), wi, wo), (x[:, :32], wi, wo), (x, wi[:128], wo), (x, wi, wo.t()), (x.cpu(), wi, wo),
                (x.t().contiguous().t(), wi, wo)):
        with pytest.raises(ValueError):
            op.forward(*bad)
    with pytest.raises(ValueError):
        op.backward(x, x, wi, wo, op.saved(5))
    with pytest.raises(gf.GatedFfnError) as e:
        op.forward(x[:0], wi, wo)
    assert e.value.code == -1
    odd = torch.zeros((4, 68), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(gf.GatedFfnError) as e:          # rows that are not 16-byte aligned
        op.forward(odd[:, :64], wi, wo)
    assert e.value.code == -1
    shifted = torch.zeros((4 * 72 + 4,), dtype=torch.bfloat16, device="cuda")[4:].view(4, 72)[:, :64]
    with pytest.raises(gf.GatedFfnError) as e:
        op.forward(shifted, wi, wo)
    assert e.value.code == -3
    with pytest.raises(ValueError):
        gf.GatedFfn(64, 128, "relu")
    with pytest.raises(ValueError):
        gf.GatedFfn(64, 128, dtype=torch.float32)
    for sizes in ((60, 128), (64, 4), (0, 128), (64, 65544)):
        with pytest.raises(gf.GatedFfnError) as e:
            gf.GatedFfn(*sizes)
        assert e.value.code == -1
    # the C entry: a missing and a small workspace
    y, hid = torch.empty_like(x), torch.empty((4, 256), dtype=torch.bfloat16, device="cuda")
    L = gf.load()
    back = [op.h, x.data_ptr(), 64, x.data_ptr(), 64, wi.data_ptr(), wo.data_ptr(), hid.data_ptr(), hid.data_ptr(),
            y.data_ptr(), 64, wi.data_ptr(), wo.data_ptr()]
    assert L.gated_ffn_backward(*back, None, 0, 4) == -2
    scratch = torch.empty((256,), dtype=torch.uint8, device="cuda")
    assert L.gated_ffn_backward(*back, scratch.data_ptr(), 256, 4) == -5
    op.status()
