"""The orthogonalised update against the binary64 oracle, through the binding.

Tolerances, in the 2-norm relative to the update's.  The update's own rounding to bfloat16 is 2^-8 of each element at most.  The
iteration: an operand's rounding is r = 2^-12 of it in the root mean square (half a step is 2^-11 at most, uniform below), the three
products of a step take five rounded operands (X twice, O twice, P and X) with off-diagonal weights that together do not exceed
those of the step's own polynomial at its steepest, p' <= 3.4445 + 3 * 4.775 * 0.3 = 7.7 in absolute terms, and what step j
leaves passes the following ones, whose slope is at most 3.9 where singular values are still small and which then share
it with a result that grows as much.  So each step counts once: 5 steps * sqrt(5) * r * 3.9 / 2 = 5.3e-3 as the bound, to which
the worst rounding of the result adds 2^-8 = 3.9e-3; for G of deficient rank the directions that are missing from it come
up from the rounding of the first steps by 3.4445^5 = 484 against the least singular value's p^5(s): doubled.
`closer` holds a full-rank G to what the diagonals' and X's precise parts are for: 1.5e-3 beyond the result's rounding,
a third of what they would cost rounded (3e-3 to 4e-2).
"""
import numpy as np
import pytest

from oracle import training as tr
from paper_2603_12145_b200 import orthogonal

pytestmark = pytest.mark.gpu

BOUND = 5.3e-3 + 2.0 ** -8


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    orthogonal.load(build_if_missing=True)
    return torch


def f64(t):
    return t.double().cpu().numpy()


def matrices(torch, seed, batch, rows, cols, dtype, rank=None, noise=1.0, scale=1.0):
    """Momentum: `rank` directions of sizes falling off over a full-rank rest of `noise` times their size."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = noise * torch.randn((batch, rows, cols), generator=g, device="cuda")
    if rank:
        u = torch.randn((batch, rows, rank), generator=g, device="cuda")
        w = torch.randn((batch, rank, cols), generator=g, device="cuda")
        v = v + (u * torch.exp(-3.0 * torch.arange(rank, device="cuda") / rank)) @ w / rank ** 0.5
    return (scale * v).to(getattr(torch, dtype))


def error(got, want):
    return np.linalg.norm(f64(got) - want) / np.linalg.norm(want)


CASES = [
    # batch, rows, cols, dtype, rank, noise
    (1, 1, 1, "float32", None, 1.0),
    (1, 1, 300, "bfloat16", None, 1.0),
    (1, 300, 1, "float16", None, 1.0),
    (3, 7, 5, "float32", None, 1.0),
    (2, 16, 48, "bfloat16", None, 1.0),
    (8, 384, 64, "float32", 4, 1.0),
    (2, 64, 200, "float16", 4, 0.3),
    (1, 130, 131, "float32", 8, 0.1),
    (3, 257, 100, "bfloat16", 8, 0.1),
    (1, 333, 777, "float32", 8, 0.03),
    (2, 576, 576, "bfloat16", 16, 0.1),
    (1, 1728, 576, "float32", 32, 0.1),
    (1, 700, 2500, "bfloat16", 32, 0.01),
    (5, 320, 512, "float16", 8, 1.0),
    (1, 2048, 2048, "bfloat16", 64, 0.3),
    (1, 4096, 1000, "float32", 64, 1.0),
    # short sides of up to 128 in one cluster: one to eight blocks, the last one's slice partly or wholly empty, either
    # way round, several groups of columns; and those whose long side is too long for it
    (1, 64, 64, "float32", 4, 1.0),
    (5, 33, 700, "bfloat16", 4, 0.3),
    (2, 700, 33, "float16", 4, 0.3),
    (1, 64, 1024, "float32", 4, 0.1),
    (1, 1100, 64, "bfloat16", 4, 1.0),
    (1, 50, 5632, "bfloat16", 4, 1.0),
    (1, 5601, 17, "float32", 4, 1.0),
    (1, 20, 6000, "bfloat16", 4, 1.0),
    (3, 128, 128, "bfloat16", 8, 0.1),
    (1, 65, 193, "float32", 8, 0.3),
    (2, 128, 1536, "float16", 8, 1.0),
    (1, 1441, 100, "bfloat16", 8, 0.1),
    (1, 90, 400, "float32", 8, 0.03),
    (1, 2000, 127, "float32", 8, 1.0),
    (40, 24, 96, "float32", 2, 1.0),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_update(torch, case):
    batch, rows, cols, dtype, rank, noise = case
    g = matrices(torch, rows + cols, batch, rows, cols, dtype, rank, noise, 1e-3)
    op = orthogonal.Orthogonal(rows, cols, dtype=getattr(torch, dtype))
    out = op.update(g)
    op.status()
    assert out.dtype is torch.bfloat16 and out.shape == g.shape
    for z in range(batch):
        want = tr.orthogonal(f64(g[z]))
        err = error(out[z], want)
        assert err <= BOUND, (z, err)
        # closer, beyond the rounding of this very result
        rounding = np.linalg.norm(f64(torch.from_numpy(want).to(torch.bfloat16)) - want) / np.linalg.norm(want)
        assert err <= np.hypot(rounding, 1.5e-3) + 1e-4, (z, err, rounding)
    assert torch.equal(op.update(g), out)
    if batch == 1:
        assert torch.equal(op.update(g[0]), out[0])


def test_deficient_rank(torch):
    for rows, cols, rank in ((200, 500, 1), (600, 300, 20)):
        g = matrices(torch, 3, 1, rows, cols, "float32", rank, 0.0)[0]
        op = orthogonal.Orthogonal(rows, cols, dtype=torch.float32)
        assert error(op.update(g), tr.orthogonal(f64(g))) <= 2 * BOUND


def test_every_direction_comes_out_alike(torch):
    """The singular values of the update of a full-rank G lie between 0.65 and 1.25 but for those that five steps
    cannot lift; the singular vectors are G's."""
    g = matrices(torch, 1, 1, 256, 1024, "float32")[0]
    op = orthogonal.Orthogonal(256, 1024, dtype=torch.float32)
    s = np.linalg.svd(f64(op.update(g)), compute_uv=False)
    assert s.min() > 0.65 and s.max() < 1.25


def test_transposed_is_the_transposed_update(torch):
    g = matrices(torch, 2, 1, 200, 456, "bfloat16", 8, 0.3)[0]
    wide, tall = orthogonal.Orthogonal(200, 456), orthogonal.Orthogonal(456, 200)
    a, b = wide.update(g), tall.update(g.t().contiguous())
    assert error(a, f64(b).T) <= BOUND


def test_sizes_do_not_matter(torch):
    """The update of a multiple: |G| from 1e-30 to 1e30 (beyond binary32's squares), eps far below."""
    g = matrices(torch, 4, 1, 96, 160, "float32")[0]
    op = orthogonal.Orthogonal(96, 160, dtype=torch.float32, eps=1e-37)
    want = tr.orthogonal(f64(g))
    for scale in (2.0 ** -100, 2.0 ** -20, 1.0, 2.0 ** 100):
        assert error(op.update(g * scale), want) <= BOUND, scale


def test_zero_matrix_and_eps(torch):
    op = orthogonal.Orthogonal(40, 60, dtype=torch.float32)
    assert (op.update(torch.zeros(40, 60, device="cuda")) == 0).all()
    g = matrices(torch, 4, 1, 40, 60, "float32", scale=1e-9)[0]          # |G| about 5e-8, half of eps
    assert error(op.update(g), tr.orthogonal(f64(g))) <= BOUND


def test_steps_and_coefficients(torch):
    g = matrices(torch, 5, 1, 100, 300, "float32")[0]
    for steps, coefficients in ((1, tr.COEFFICIENTS), (2, (1.5, -0.5, 0.0)), (12, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5))):
        op = orthogonal.Orthogonal(100, 300, dtype=torch.float32, steps=steps, coefficients=coefficients)
        want = tr.orthogonal(f64(g), steps=steps, coefficients=coefficients)
        assert error(op.update(g), want) <= BOUND, (steps, coefficients)


def test_nan_stays_in_its_matrix(torch):
    g = matrices(torch, 6, 4, 128, 72, "bfloat16")
    op = orthogonal.Orthogonal(128, 72)
    clean = op.update(g)
    g[1, 100, 3] = float("nan")
    g[3, 0, 71] = float("inf")
    out = op.update(g)
    assert torch.isnan(out[1]).all() and torch.isnan(out[3]).all()
    assert torch.equal(out[0], clean[0]) and torch.equal(out[2], clean[2])


def test_strides_and_surroundings(torch):
    """G in columns of a wider array, transposed batches, one matrix for all; the update into a part of an array."""
    for rows, cols in ((50, 72), (72, 50), (33, 35)):
        op = orthogonal.Orthogonal(rows, cols)
        g = matrices(torch, 7, 3, rows, cols, "bfloat16")
        want = op.update(g)
        wide = torch.full((3, rows, cols + 9), float("nan"), dtype=g.dtype, device="cuda")
        wide[:, :, 5:5 + cols] = g
        assert torch.equal(op.update(wide[:, :, 5:5 + cols]), want)
        inner = g.transpose(0, 1).contiguous().transpose(0, 1)
        assert torch.equal(op.update(inner), want)
        assert torch.equal(op.update(g[1:2].expand(3, rows, cols)), want[1:2].expand(3, rows, cols))
        big = torch.full((3, rows + 2, cols + 7), 7.0, dtype=torch.bfloat16, device="cuda")
        op.update(g, out=big[:, 1:1 + rows, 3:3 + cols])
        assert torch.equal(big[:, 1:1 + rows, 3:3 + cols], want)
        big[:, 1:1 + rows, 3:3 + cols] = 7.0
        assert (big == 7.0).all()


def test_two_handles_side_stream_and_graph(torch):
    a, b = orthogonal.Orthogonal(128, 320), orthogonal.Orthogonal(200, 136)
    g, h = matrices(torch, 8, 2, 128, 320, "bfloat16"), matrices(torch, 9, 1, 200, 136, "bfloat16")
    want = [a.update(g), b.update(h)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = a.update(g)
    second = b.update(h)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, want[0]) and torch.equal(second, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = [a.update(g), b.update(h)]
    g.copy_(matrices(torch, 10, 2, 128, 320, "bfloat16"))
    graph.replay()
    got = [v.clone() for v in captured]
    assert torch.equal(got[0], a.update(g)) and torch.equal(got[1], want[1])
    a.status()
    b.status()


def test_two_streams_at_once(torch):
    """Updates that take the whole device, on two streams without an order between them."""
    sizes = ((1728, 576), (1024, 2048), (300, 300), (64, 700))
    ops = [orthogonal.Orthogonal(m, n) for m, n in sizes]
    gs = [matrices(torch, 20 + i, 1, m, n, "bfloat16", 8, 0.3)[0] for i, (m, n) in enumerate(sizes)]
    want = [op.update(g) for op, g in zip(ops, gs)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(w) for w in want] for _ in range(6)]
    torch.cuda.synchronize()
    for k, out in enumerate(outs):
        for i, op in enumerate(ops):
            with torch.cuda.stream(streams[(i + k) % 2]):
                op.update(gs[i], out=out[i])
    torch.cuda.synchronize()
    for op in ops:
        op.status()
    for out in outs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("rows,cols", [(100, 60), (200, 300)])
def test_least_eps(torch, rows, cols):
    """Norms whose inverse is beyond binary32: no zero times infinity."""
    op = orthogonal.Orthogonal(rows, cols, dtype=torch.float32, eps=2.0 ** -149)
    assert (op.update(torch.zeros(rows, cols, device="cuda")) == 0).all()
    g = matrices(torch, 4, 1, rows, cols, "float32")[0]
    want = tr.orthogonal(f64(g))
    assert error(op.update(g), want) <= BOUND
    small = g * 2.0 ** -124                       # some are subnormal: taken as they are
    assert error(op.update(small), tr.orthogonal(f64(small), eps=2.0 ** -149)) <= BOUND


def test_refusals(torch):
    op = orthogonal.Orthogonal(40, 60)
    g = matrices(torch, 1, 2, 40, 60, "bfloat16")
    for bad in (g.float(), g[:, :39], g[:, :, :59], g.cpu(), g.transpose(1, 2), g[0, 0], g[None]):
        with pytest.raises(ValueError):
            op.update(bad)
    for out in (g.float(), g[:1], g.transpose(1, 2)):
        with pytest.raises(ValueError):
            op.update(g, out=out)
    for call in (lambda: op.update(g[:0]), lambda: op.update(g, out=torch.empty_like(g[:1]).expand(2, 40, 60)),
                 lambda: op.update(g[0], out=torch.empty_like(g[0, :1]).expand(40, 60))):
        with pytest.raises(orthogonal.OrthogonalError) as ei:
            call()
        assert ei.value.code == -1
    for kw in (dict(rows=0, cols=4), dict(rows=4, cols=65537), dict(rows=4, cols=4, steps=0), dict(rows=4, cols=4, steps=33),
               dict(rows=4, cols=4, eps=0.0), dict(rows=4, cols=4, eps=float("inf")),
               dict(rows=4, cols=4, coefficients=(float("nan"), 0.0, 0.0))):
        with pytest.raises(orthogonal.OrthogonalError) as ei:
            orthogonal.Orthogonal(**kw)
        assert ei.value.code == -1
    with pytest.raises(ValueError):
        orthogonal.Orthogonal(4, 4, dtype=torch.float64)
