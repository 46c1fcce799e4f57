"""The gated feed-forward block over the loops that large calls run in (several tiles per pair, in the second
accumulator buffer and staged blocks used again; tiles of 192 columns), the planes that keep g and u, and the
block inside a CUDA graph.  test_host_calls.py checks that TILES cases are cut as they say.

Kept g and u: a binary32 accumulation of K terms (within K 2^-23 of the sum of absolute terms), cut off to 24
bits, of which 15 are behind the leading one of the fraction: below 2^-15 relative."""
import numpy as np
import pytest

from oracle import sequence as seq
from paper_2603_12145_b200 import gated_ffn as gf

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -23
UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}

# rows, model, hidden, activation, dtype; and pairs at work in the forward and in the slope product with their rounds of
# tiles (2,600 rows are eleven tiles; 1,032 units nine tiles of 128 forward, six of 192 backward)
TILES = [(2600, 64, 1032, "silu", "bfloat16", (74, 2), (66, 1)), (5200, 72, 1032, "gelu", "float16", (74, 3), (74, 2)),
         (5200, 40, 520, "silu", "float16", (74, 2), (63, 1))]


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    gf.load(build_if_missing=True)
    return torch


def device(torch, a, dtype):
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda().to(getattr(torch, dtype))
    return t, t.double().cpu().numpy()


def check(name, got, want, tol):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, first at %s: got %r want %r tol %r" % (
        name, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], np.broadcast_to(tol, got.shape)[bad][0])


def planes(torch, kept, n, hidden):
    """What the library keeps, [n][2][hidden] in binary64: 16 upper bits in one plane, 8 more in another, whose rows
    are whole 16-byte pieces and which begins 256-byte aligned."""
    wide, first = (hidden + 15) // 16 * 16, (n * hidden * 4 + 255) // 256 * 256
    assert kept.numel() == first + n * 2 * wide
    upper = kept[:n * hidden * 4].view(torch.int16).view(n, 2, hidden).to(torch.int32) & 0xFFFF
    lower = kept[first:].view(n, 2, wide)[:, :, :hidden].to(torch.int32)
    return ((upper << 16) | (lower << 8)).view(torch.float32).double().cpu().numpy()


def operands(seed, n, model, hidden):
    r = np.random.Generator(np.random.PCG64(seed))
    return (r.standard_normal((n, model)), r.standard_normal((2 * hidden, model)) * model ** -0.5,
            r.standard_normal((model, hidden)) * hidden ** -0.5, r.standard_normal((n, model)))


@pytest.mark.parametrize("case", TILES + [(5, 200, 136, "silu", "float16"), (33, 64, 72, "gelu", "bfloat16")], ids=str)
def test_forward_keeps_the_preactivations(torch, case):
    n, model, hidden, activation, dtype = case[:5]
    x, w_in, w_out, _ = operands(n, n, model, hidden)
    (xd, x), (wi, w_in), (wo, w_out) = device(torch, x, dtype), device(torch, w_in, dtype), device(torch, w_out, dtype)
    op = gf.GatedFfn(model, hidden, activation, getattr(torch, dtype))
    kept = op.saved(n)
    kept[0].fill_(255)
    y = op.forward(xd, wi, wo, saved=kept)
    op.status()
    want_y, pre, hid = seq.gated_ffn(x, w_in, w_out, activation)
    e_in = model * EPS * (np.abs(x) @ np.abs(w_in).T)
    check("g and u", planes(torch, kept[0], n, hidden).reshape(n, 2 * hidden), pre, 1.1 * e_in + 2.0 ** -15 * np.abs(pre))
    # hidden: rounded to the type from the unrounded g and u (|act'| <= 1.13)
    u, least = UNIT[dtype], (2.0 ** -24 if dtype == "float16" else 0.0)
    act = np.abs(seq.ACTIVATIONS[activation][0](pre[:, :hidden]))
    e_h = 1.1 * (u * np.abs(hid) + 1.2 * (np.abs(pre[:, hidden:]) * e_in[:, :hidden] + act * e_in[:, hidden:]) + 2.0 ** -21 * np.abs(hid)) + least
    check("hidden", kept[1].double().cpu().numpy(), hid, e_h)
    check("y", y.double().cpu().numpy(), want_y,
          1.1 * (e_h @ np.abs(w_out).T + hidden * EPS * (np.abs(hid) @ np.abs(w_out).T)) + u * np.abs(want_y) + least)
    assert torch.equal(op.forward(xd, wi, wo), y)


@pytest.mark.parametrize("case", [(2600, 1032, "silu"), (300, 1032, "gelu"), (5200, 136, "gelu"), (600, 776, "silu")], ids=str)
def test_backward_reads_all_kept_bits(torch, case):
    """dg and du one by one: with W_in the unit matrix, dx is [dg | du].  dhidden is exact (small multiples of powers of
    two), g and u are given with all their 24 bits; a wrong or missing lower byte moves them by up to 2^-7.

        dg = dhidden u act'(g),  du = dhidden act(g):  one rounding to binary16 and a few of binary32, of which the
    slope's add up to 2^-20 of the sum of absolute terms (the sigmoid and its products)."""
    n, hidden, activation = case
    model = 2 * hidden
    r = np.random.Generator(np.random.PCG64(n))
    dy, w_out = r.integers(-2, 3, (n, model)) / 4.0, r.integers(-2, 3, (model, hidden)) / 16.0
    pre = r.standard_normal((n, 2, hidden)).astype(np.float32).view(np.uint32) & 0xFFFFFF00
    op = gf.GatedFfn(model, hidden, activation, torch.float16)
    wide, first = (hidden + 15) // 16 * 16, (n * hidden * 4 + 255) // 256 * 256
    kept, hid = op.saved(n)
    kept.fill_(255)
    kept[:n * hidden * 4] = torch.from_numpy((pre >> 16).astype(np.uint16).view(np.uint8).reshape(-1)).cuda()
    kept[first:].view(n, 2, wide)[:, :, :hidden] = torch.from_numpy(((pre >> 8) & 0xFF).astype(np.uint8)).cuda()
    pre = pre.view(np.float32).astype(np.float64)
    assert np.array_equal(planes(torch, kept, n, hidden), pre)
    dev = [device(torch, v, "float16")[0] for v in (dy, np.zeros((n, model)), np.eye(model), w_out)]
    dx, _, _ = op.backward(*dev, (kept, hid.zero_()))
    op.status()
    g, u, dh = pre[:, 0], pre[:, 1], dy @ w_out
    act, slope = seq.ACTIVATIONS[activation]
    want = np.concatenate([dh * u * slope(g), dh * act(g)], axis=1)
    mag = np.concatenate([np.abs(dh * u) * 1.2 * (1 + np.abs(g)), np.abs(dh * g)], axis=1)
    check("dg and du", dx.double().cpu().numpy(), want, 2.0 ** -11 * np.abs(want) + 2.0 ** -20 * mag + 2.0 ** -24)


@pytest.mark.parametrize("case", TILES, ids=str)
def test_gradients_over_several_tiles(torch, case):
    """Against the definition in the norm: dg, du and hidden are rounded to the type (u each) and so is the result;
    independent roundings of u at most, u / sqrt(3) in the mean square, add up to sqrt(2) of that, and twice this bound leaves
    room for the distribution of the last bits."""
    n, model, hidden, activation, dtype = case[:5]
    x, w_in, w_out, dy = operands(n + 1, n, model, hidden)
    (xd, x), (wi, w_in), (wo, w_out), (dyd, dy) = [device(torch, v, dtype) for v in (x, w_in, w_out, dy)]
    op = gf.GatedFfn(model, hidden, activation, getattr(torch, dtype))
    kept = op.saved(n)
    op.forward(xd, wi, wo, saved=kept)
    got = op.backward(dyd, xd, wi, wo, kept)
    again = op.backward(dyd, xd, wi, wo, kept)
    op.status()
    for name, g, s, w in zip(("dx", "dw_in", "dw_out"), got, again, seq.gated_ffn_grad(dy, x, w_in, w_out, activation)):
        off = np.linalg.norm(g.double().cpu().numpy() - w) / np.linalg.norm(w)
        assert off <= 2 * (2 / 3) ** 0.5 * UNIT[dtype], (name, off)
        worst = np.abs(g.double().cpu().numpy() - w).max() / np.abs(w).max()
        assert worst <= 8 * UNIT[dtype], (name, worst)       # no tile of its own is off
        assert torch.equal(g, s)


@pytest.mark.parametrize("n", [1, 40, 300])
def test_block_replays_from_a_cuda_graph(torch, n):
    """Forward and backward captured once and replayed on changing inputs: the bits of eager calls."""
    model, hidden = 136, 264
    values = [[device(torch, v, "bfloat16")[0] for v in operands(seed, n, model, hidden)] for seed in range(3)]
    op = gf.GatedFfn(model, hidden, "gelu")
    held, kept = [v.clone() for v in values[0]], op.saved(n)

    def run(v, buffers):
        y = op.forward(*v[:3], saved=buffers)
        return (y,) + op.backward(v[3], *v[:3], buffers)

    run(held, op.saved(n))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(held, kept)
    for v in values:
        for h, w in zip(held, v):
            h.copy_(w)
        graph.replay()
        want = run(v, op.saved(n))
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    op.status()
