"""The layer norm against the binary64 oracle, through the binding.

Tolerances.  u = 2^-24 is binary32's unit roundoff, u_T that of the type (2^-8, 2^-11, 2^-24): half a step, relative.  A
row's sums are chains of at most 32 terms per thread and 10 joins: K = 48 roundings with those of the terms.  With S the
mean of |s| over the row, q = 1 / standard deviation, z = (s - m) q:

    the mean is off by K u S, a z by  dz = K u (q S + |z|)   (its own difference, the mean, half the variance's K + 4)
    y:  u_T |y| + |w| dz + 4 u (|z w| + |b|)
    dx: u_T |dx| + q [K u (|c| + mean|c| + |z| mean|c z|) + dz mean|c z| + |z| mean(|c| dz)] + K u |dx - dsum| + u |dsum|
    dw: sum |dy| dz + R u sum|dy z|    db: R u sum|dy|    R = min(rows, 600) + 16 roundings along the rows

The residual's sum is one rounding of a binary32 sum and is compared bit by bit.
"""
import numpy as np
import pytest

from oracle import training as tr
from paper_2603_12145_b200 import layer_norm

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
UNIT = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
K = 48


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    layer_norm.load(build_if_missing=True)
    return torch


def f64(t):
    return t.double().cpu().numpy()


def make(torch, seed, n, width, dtype, layout="dense", offset=1.0, device="cuda"):
    """Rows of the type.  layout: "dense", "wide" (columns of a wider array at an odd offset), "pitch" (rows of whole
    vectors apart)."""
    g = torch.Generator(device=device).manual_seed(seed)
    v = (torch.randn((n, width), generator=g, device=device) + offset).to(getattr(torch, dtype))
    if layout == "wide":
        big = torch.full((n, width + 5), float("nan"), dtype=v.dtype, device=device)
        big[:, 3:3 + width] = v
        v = big[:, 3:3 + width]
    elif layout == "pitch":
        big = torch.full((n, width + 16), float("nan"), dtype=v.dtype, device=device)
        big[:, :width] = v
        v = big[:, :width]
    return v


def near(name, got, want, tol, dtype):
    got = f64(got)
    tol = tol + (2.0 ** -25 if dtype == "float16" else 1e-37)          # half of the least subnormal number
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, first at %s: got %r want %r tol %r" % (
        name, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], np.broadcast_to(tol, got.shape)[bad][0])


def check_forward(s, y, w, b, eps, dtype):
    want, mean, q = tr.norm(s, w, b, eps)
    z = (s - mean[:, None]) * q[:, None]
    dz = K * U * (q * np.abs(s).mean(axis=1))[:, None] + K * U * np.abs(z)
    aw = np.ones(s.shape[1]) if w is None else np.abs(w)
    ab = np.zeros(s.shape[1]) if b is None else np.abs(b)
    near("y", y, want, UNIT[dtype] * np.abs(want) + aw * dz + 4 * U * (np.abs(z) * aw + ab), dtype)


def check_backward(s, dy, w, dsum, eps, dtype, dx, dw, db):
    want_dx, want_dw, want_db = tr.norm_grad(dy, s, w, dsum, eps)
    _, mean, q = tr.norm(s, eps=eps)
    z = np.abs((s - mean[:, None]) * q[:, None])
    q = q[:, None]
    dz = K * U * (q * np.abs(s).mean(axis=1, keepdims=True) + z)
    c = np.abs(dy if w is None else dy * w)
    cz = (c * z).mean(axis=1, keepdims=True)
    ads = 0.0 if dsum is None else np.abs(dsum)
    tol = (UNIT[dtype] * np.abs(want_dx) + U * ads + K * U * np.abs(want_dx - (0.0 if dsum is None else dsum))
           + q * (K * U * (c + c.mean(axis=1, keepdims=True) + z * cz) + dz * cz + z * (c * dz).mean(axis=1, keepdims=True)))
    near("dx", dx, want_dx, tol, dtype)
    if dw is not None:
        rows = (min(len(s), 600) + 16) * U
        near("dw", dw, want_dw, (np.abs(dy) * dz).sum(axis=0) + rows * (np.abs(dy) * z).sum(axis=0), "float32")
        near("db", db, want_db, rows * np.abs(dy).sum(axis=0), "float32")


CASES = [
    # rows, width, dtype, layout, residual, weights
    (1, 1, "float32", "dense", False, True),          # one element: z = 0
    (1, 7, "bfloat16", "dense", True, True),
    (5, 8, "bfloat16", "dense", True, False),         # one vector: three of four lanes without
    (3, 64, "float16", "pitch", True, True),
    (33, 96, "float32", "dense", False, True),
    (9, 100, "float32", "wide", True, True),
    (200, 128, "bfloat16", "dense", True, True),
    (130, 255, "float16", "wide", True, True),
    (17, 257, "bfloat16", "dense", False, True),      # single elements, a block per row
    (64, 576, "bfloat16", "dense", True, True),
    (70, 512, "float32", "pitch", True, True),
    (40, 1024, "bfloat16", "dense", True, False),
    (21, 1003, "float32", "dense", True, True),
    (19, 1152, "float16", "dense", False, True),      # a block per row: 64 threads with three vectors
    (6, 5001, "bfloat16", "wide", True, True),        # 16 elements per thread
    (5, 6152, "float32", "dense", True, True),        # four vectors of four
    (7, 8192, "bfloat16", "dense", True, True),
    (4, 8192, "float32", "dense", False, True),
    (3, 8191, "float32", "dense", False, True),
    (20000, 72, "bfloat16", "dense", True, True),     # several rows per group
    (3000, 2048, "float16", "dense", True, True),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward_and_backward(torch, case):
    n, width, dtype, layout, residual, weights = case
    op = layer_norm.LayerNorm(width, eps=1e-5, dtype=getattr(torch, dtype))
    x, dy = make(torch, 1, n, width, dtype, layout), make(torch, 2, n, width, dtype, layout, 0.0)
    r = make(torch, 3, n, width, dtype, layout, 0.0) if residual else None
    d = make(torch, 4, n, width, dtype, layout, 0.0) if residual else None
    w = make(torch, 5, 1, width, "float32")[0] if weights else None
    b = make(torch, 6, 1, width, "float32", offset=0.0)[0] if weights else None
    saved = op.saved(n)
    out = make(torch, 9, n, width, dtype, layout)      # results in the same kind of rows
    if residual:
        y, s = op.forward(x, w, b, residual=r, saved=saved, out=out)
        assert torch.equal(s, (x.float() + r.float()).to(x.dtype))
    else:
        y, s = op.forward(x, w, b, saved=saved, out=out), x
    assert y is out
    dx, dw, db = op.backward(dy, s, w, saved, dsum=d)
    torch.cuda.synchronize()
    s64, w64, b64 = f64(s), None if w is None else f64(w), None if b is None else f64(b)
    check_forward(s64, y, w64, b64, 1e-5, dtype)
    check_backward(s64, f64(dy), w64, None if d is None else f64(d), 1e-5, dtype, dx, dw, db)
    # without weights' gradients the rows' is the same, and so are the bits of a second call
    again = op.backward(dy, s, w, saved, dsum=d)
    alone = op.backward(dy, s, w, saved, dsum=d, want_params=False)
    assert torch.equal(alone[0], dx) and alone[1] is None and alone[2] is None
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))


# The widths at which the share of a thread changes: whole rounds of a warp with a rest by twos and fours, up to three
# vectors per lane (of binary32 four), blocks of 64 threads and more.
EDGES = [
    (37, 264, "bfloat16"), (37, 320, "float16"), (45, 384, "bfloat16"), (300, 576, "float16"), (41, 640, "bfloat16"),
    (40, 768, "bfloat16"), (23, 776, "bfloat16"), (23, 832, "float16"), (19, 1536, "bfloat16"), (19, 1544, "float16"),
    (11, 4096, "bfloat16"), (9, 4104, "float16"), (31, 256, "float32"), (31, 260, "float32"), (29, 384, "float32"),
    (29, 388, "float32"), (27, 516, "float32"), (17, 1028, "float32"), (13, 2052, "float32"), (7, 4100, "float32"),
    (33, 128, "float32"), (21, 129, "bfloat16"), (15, 513, "float32"), (12, 2049, "float16"), (9, 4097, "bfloat16"),
]


@pytest.mark.parametrize("case", EDGES, ids=str)
def test_widths_between_shares(torch, case):
    n, width, dtype = case
    op = layer_norm.LayerNorm(width, eps=1e-5, dtype=getattr(torch, dtype))
    x, r = make(torch, 1, n, width, dtype), make(torch, 2, n, width, dtype, offset=-0.5)
    dy, dsum = make(torch, 3, n, width, dtype, offset=0.0), make(torch, 4, n, width, dtype, offset=0.0)
    w, b = make(torch, 5, 1, width, "float32")[0], make(torch, 6, 1, width, "float32")[0]
    saved = op.saved(n)
    y, total = op.forward(x, w, b, residual=r, saved=saved)
    assert torch.equal(total, x + r)
    check_forward(f64(total), y, f64(w), f64(b), 1e-5, dtype)
    dx, dw, db = op.backward(dy, total, w, saved, dsum=dsum)
    check_backward(f64(total), f64(dy), f64(w), f64(dsum), 1e-5, dtype, dx, dw, db)
    alone = op.backward(dy, total, w, saved, dsum=dsum, want_params=False)
    assert torch.equal(alone[0], dx)


# Rows that begin and end between boundaries of 16 bytes: many remainders, widths at which the share or the way to read them changes,
# several rows per thread, and the widest.
BETWEEN = [
    (5, 1, "bfloat16"), (9, 2, "float16"), (11, 7, "bfloat16"), (20, 9, "float16"), (40, 33, "bfloat16"), (20000, 65, "bfloat16"),
    (33, 66, "float16"), (35, 129, "bfloat16"), (37, 250, "bfloat16"), (9000, 255, "bfloat16"), (3000, 577, "float16"),
    (19, 759, "bfloat16"), (19, 763, "bfloat16"), (23, 1001, "float16"), (1300, 2001, "bfloat16"), (17, 2045, "bfloat16"),
    (15, 3067, "float16"), (1000, 5001, "bfloat16"), (9, 8177, "float16"), (9, 8179, "bfloat16"), (7, 8191, "float16"),
    (20000, 35, "float32"), (31, 1, "float32"), (31, 5, "float32"), (3000, 131, "float32"), (33, 254, "float32"),
    (2000, 509, "float32"), (21, 511, "float32"),
]


@pytest.mark.parametrize("layout", ["dense", "wide"])
@pytest.mark.parametrize("case", BETWEEN, ids=str)
def test_rows_between_boundaries(torch, case, layout):
    n, width, dtype = case
    op = layer_norm.LayerNorm(width, eps=1e-5, dtype=getattr(torch, dtype))
    x, r, dy, dsum = (make(torch, seed, n, width, dtype, layout, offset=0.5) for seed in (1, 2, 3, 4))
    w, b = make(torch, 5, 1, width, "float32")[0], make(torch, 6, 1, width, "float32")[0]
    room = [make(torch, 7, n, width, dtype, layout) for _ in range(3)]
    saved = op.saved(n)
    y, total = op.forward(x, w, b, residual=r, saved=saved, out=room[0], total=room[1])
    assert torch.equal(total, x + r)
    check_forward(f64(total), y, f64(w), f64(b), 1e-5, dtype)
    dx, dw, db = op.backward(dy, total, w, saved, dsum=dsum, out=room[2])
    check_backward(f64(total), f64(dy), f64(w), f64(dsum), 1e-5, dtype, dx, dw, db)
    if layout == "wide":                      # nothing beside the columns
        for v in room:
            whole = v._base
            assert torch.isnan(whole[:, :3]).all() and torch.isnan(whole[:, 3 + width:]).all()
    again = op.backward(dy, total, w, saved, dsum=dsum, out=make(torch, 7, n, width, dtype, layout))
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))


@pytest.mark.parametrize("width", [8, 64, 256, 576, 768, 1024, 8192])
@pytest.mark.parametrize("n", [1, 2, 3])
def test_few_rows(torch, n, width):
    """Fewer rows than a thread, a warp or a block goes through at a time."""
    op = layer_norm.LayerNorm(width, eps=1e-5)
    x, r, dy = (make(torch, seed, n, width, "bfloat16", offset=0.5) for seed in (1, 2, 3))
    w, b = make(torch, 5, 1, width, "float32")[0], make(torch, 6, 1, width, "float32")[0]
    room = [torch.full((n + 2, width), 7.0, dtype=x.dtype, device="cuda") for _ in range(3)]
    saved = op.saved(n)
    y, total = op.forward(x, w, b, residual=r, saved=saved, out=room[0][:n], total=room[1][:n])
    assert torch.equal(total, x + r)
    check_forward(f64(total), y, f64(w), f64(b), 1e-5, "bfloat16")
    dx, dw, db = op.backward(dy, total, w, saved, out=room[2][:n])
    check_backward(f64(total), f64(dy), f64(w), None, 1e-5, "bfloat16", dx, dw, db)
    assert all((v[n:] == 7.0).all() for v in room)


def test_large_offset_and_constant_rows(torch):
    """Rows far from zero lose nothing to cancellation beyond the mean's rounding; a constant row is all b."""
    op = layer_norm.LayerNorm(576, dtype=torch.float32)
    x = make(torch, 1, 40, 576, "float32", offset=3000.0)
    x[7] = 5.0
    b = make(torch, 2, 1, 576, "float32")[0]
    y = op.forward(x, None, b)
    check_forward(f64(x), y, None, f64(b), 1e-5, "float32")
    assert torch.equal(y[7], b)


def test_in_place(torch):
    """The stream updated where it is, and gradients over the incoming ones."""
    for width, dtype in ((576, torch.bfloat16), (101, torch.float32), (4096, torch.float16)):
        op = layer_norm.LayerNorm(width, dtype=dtype)
        name = str(dtype).split(".")[1]
        x, r = make(torch, 1, 300, width, name), make(torch, 2, 300, width, name)
        saved = op.saved(300)
        y, s = op.forward(x, residual=r, saved=saved)
        x2, r2 = x.clone(), r.clone()
        y2, s2 = op.forward(x2, residual=r, total=x2)
        assert s2 is x2 and torch.equal(x2, s) and torch.equal(y2, y)
        y3, s3 = op.forward(x, residual=r2, total=r2)
        assert s3 is r2 and torch.equal(r2, s) and torch.equal(y3, y)
        z = s.clone()
        assert torch.equal(op.forward(z, out=z), op.forward(s))
        dy, d = make(torch, 3, 300, width, name), make(torch, 4, 300, width, name)
        want = op.backward(dy, s, None, saved, dsum=d)
        for k in range(2):
            dy2, d2 = dy.clone(), d.clone()
            got = op.backward(dy2, s, None, saved, dsum=d2, out=(dy2, d2)[k])
            assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_nan_and_infinity_stay_in_their_rows(torch):
    for width in (64, 777, 2048):
        op = layer_norm.LayerNorm(width, dtype=torch.bfloat16)
        x = make(torch, 1, 50, width, "bfloat16")
        clean = op.forward(x)
        x[3, width // 2] = float("nan")
        x[11, 0] = float("inf")
        x[49, width - 1] = float("-inf")
        y = op.forward(x)
        hit = torch.zeros(50, dtype=torch.bool, device="cuda")
        hit[[3, 11, 49]] = True
        assert torch.isnan(y[hit]).all() and torch.equal(y[~hit], clean[~hit])


def test_one_row_for_all(torch):
    """Stride 0: a row that serves as every row's residual or incoming gradient."""
    op = layer_norm.LayerNorm(200, dtype=torch.bfloat16)
    x, r = make(torch, 1, 30, 200, "bfloat16"), make(torch, 2, 1, 200, "bfloat16")
    saved = op.saved(30)
    y, s = op.forward(x, residual=r.expand(30, 200), saved=saved)
    y2, s2 = op.forward(x, residual=r.expand(30, 200).contiguous())
    assert torch.equal(y, y2) and torch.equal(s, s2)
    g = op.backward(r.expand(30, 200), s, None, saved, dsum=r.expand(30, 200))
    c = r.expand(30, 200).contiguous()
    assert all(torch.equal(p, q) for p, q in zip(g, op.backward(c, s, None, saved, dsum=c)))


def test_rows_beyond_32_bit_offsets(torch):
    """Rows 2^31 and more elements from the first."""
    rows, width, stride = 3, 1152, 2 ** 30 + 8
    big = torch.empty((2 * stride + width,), dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((rows, width), (stride, 1))
    v = make(torch, 1, rows, width, "bfloat16")
    x.copy_(v)
    op = layer_norm.LayerNorm(width)
    saved = op.saved(rows)
    y = op.forward(x, saved=saved)
    assert torch.equal(y, op.forward(v))
    want = op.backward(v, v, None, saved)
    op.backward(v, x, None, saved, out=x)
    assert torch.equal(x, want[0])


def test_rows_behind_and_columns_beside_stay(torch):
    op = layer_norm.LayerNorm(72, dtype=torch.bfloat16)
    big = torch.full((20, 96), 7.0, dtype=torch.bfloat16, device="cuda")
    x = make(torch, 1, 13, 72, "bfloat16")
    saved = op.saved(13)
    op.forward(x, saved=saved, out=big[:13, :72])
    assert (big[13:] == 7.0).all() and (big[:, 72:] == 7.0).all()
    big.fill_(7.0)
    op.backward(x, x, None, saved, out=big[:13, 16:88])
    assert (big[13:] == 7.0).all() and (big[:, :16] == 7.0).all() and (big[:, 88:] == 7.0).all()


def test_side_stream_and_graph(torch):
    op = layer_norm.LayerNorm(576)
    x, r, w = make(torch, 1, 500, 576, "bfloat16"), make(torch, 2, 500, 576, "bfloat16"), make(torch, 3, 1, 576, "float32")[0]
    saved = op.saved(500)

    def run():
        y, s = op.forward(x, w, None, residual=r, saved=saved)
        return (y, s) + op.backward(r, s, w, saved, dsum=x)

    want = [v.clone() for v in run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    x2 = make(torch, 7, 500, 576, "bfloat16")
    x.copy_(x2)
    graph.replay()
    first = [v.clone() for v in captured]
    want = run()
    assert all(torch.equal(a, b) for a, b in zip(first, want))


def test_refusals(torch):
    op = layer_norm.LayerNorm(64)
    x = make(torch, 1, 4, 64, "bfloat16")
    saved = op.saved(4)
    w = torch.ones(64, device="cuda")
    for bad in (x.float(), x[:, :63], x.t(), x.cpu(), x[:, ::2], x[0]):
        with pytest.raises((ValueError, IndexError)):
            op.forward(bad)
    with pytest.raises(ValueError):
        op.forward(x, w.to(torch.bfloat16))
    with pytest.raises(ValueError):
        op.forward(x, residual=x[:3])
    with pytest.raises(ValueError):
        op.forward(x, total=x)
    with pytest.raises(ValueError):
        op.forward(x, saved=op.saved(5))
    with pytest.raises(ValueError):
        op.backward(x, x, w, saved, dsum=x.float())
    for call in (lambda: op.forward(x[:0]), lambda: op.forward(x, out=x[:1].expand(4, 64)),
                 lambda: op.backward(x[:0], x[:0], None, op.saved(0))):
        with pytest.raises(layer_norm.LayerNormError) as ei:
            call()
        assert ei.value.code == -1
    for width, eps in ((0, 1e-5), (8193, 1e-5), (64, 0.0), (64, float("nan")), (64, float("inf")), (64, -1.0)):
        with pytest.raises(layer_norm.LayerNormError) as ei:
            layer_norm.LayerNorm(width, eps=eps)
        assert ei.value.code == -1
    with pytest.raises(ValueError):
        layer_norm.LayerNorm(64, dtype=torch.float64)
