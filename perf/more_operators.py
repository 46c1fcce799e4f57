"""The cases on which the operators of a policy's training step are measured: layer norm with its residual addition
(layer_norm.py), the gated linear recurrence (gated_recurrence.py: whole sequences, their gradients, single tokens) and
the orthogonalised update of a weight matrix (orthogonal.py).

`run` computes a case with the package's kernels where `own` is true and otherwise from elementary torch operations in
binary32; `exact` evaluates the operators' definitions in binary64.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DEVICE = "cuda"
EPS = 1e-5                                   # of the norm
STEPS, NS_A, NS_B, NS_C, NS_EPS = 5, 3.4445, -4.7750, 2.0315, 1e-7


# ---- cases --------------------------------------------------------------------------

def _norm(name, kind, rows, width, dtype="bf16", residual=True):
    return {"name": name, "op": kind, "rows": rows, "width": width, "dtype": dtype, "residual": residual}


def _rec(name, kind, batch, time, channels, dtype="bf16", layout="batch", reset=False, carry=False):
    return {"name": name, "op": kind, "batch": batch, "time": time, "channels": channels, "dtype": dtype,
            "layout": layout, "reset": reset, "carry": carry}


def _orth(name, batch, rows, cols, dtype="bf16"):
    return {"name": name, "op": "orthogonal", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype}


def listed():
    return [
        # the norm of one agent step at 64 envs, in front of a layer of the policy's 576 units
        _norm("norm_rows_64", "norm_forward", 64, 576),
        # training on a rollout of 512 envs x 128 steps: the residual stream goes through, its gradient comes back
        _norm("norm_train_65536", "norm_train", 65536, 576),
        # training at generic width, the first norm of a network: nothing to add
        _norm("norm_train_wide", "norm_train", 8192, 8192, residual=False),
        # odd sizes in binary32: rows that no vector divides
        _norm("norm_train_odd_f32", "norm_train", 777, 1003, dtype="f32"),
        # one agent step of a few envs with a recurrence twice as wide as the policy's 576 units
        _rec("recurrence_step_64", "recurrence_step", 64, 1, 1152, reset=True),
        # one agent step of a large batch of envs: the recurrent state passes through memory once
        _rec("recurrence_step_16384", "recurrence_step", 16384, 1, 1152, reset=True),
        # one long prompt: a single row, whose time axis is all there is to split
        _rec("recurrence_prompt_1x8192", "recurrence_forward", 1, 8192, 2048),
        # training on a rollout as the env writes it: time-major, episodes end inside, state carried in
        _rec("recurrence_train_512x128", "recurrence_train", 512, 128, 1152, layout="time", reset=True, carry=True),
        # training in binary32 on odd sizes: few rows, channels that no vector divides
        _rec("recurrence_train_odd_f32", "recurrence_train", 3, 777, 331, dtype="f32", reset=True),
        # one weight of eight narrow layers: 64 units, a feed-forward block's two projections
        _orth("orthogonal_8x384x64", 8, 384, 64, dtype="f32"),
        # the input weights of a 576-unit GRU's three gates
        _orth("orthogonal_1728x576", 1, 1728, 576, dtype="f32"),
        # a projection of generic width
        _orth("orthogonal_2048x8192", 1, 2048, 8192),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_forward", "norm_train", "norm_train", "recurrence_step", "recurrence_forward",
                     "recurrence_train", "recurrence_train", "orthogonal", "orthogonal"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op.startswith("norm"):
        width = _log_int(rng, 33, 8192)
        if rng.random() < 0.5:
            width = (width + 7) // 8 * 8
        rows = _log_int(rng, 1, min(65536, 8192 * 8192 // (width * (2 if dtype == "f32" else 1))))
        return _norm(None, op, rows, width, dtype, rng.random() < 0.5)
    if op == "orthogonal":
        rows, cols = _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)
        if rng.random() < 0.5:
            rows, cols = (rows + 7) // 8 * 8, (cols + 7) // 8 * 8
        most = 2048 * 2048 * 8192 // (min(rows, cols) ** 2 * max(rows, cols))
        return _orth(None, _log_int(rng, 1, max(1, min(16, most))), rows, cols, dtype)
    channels = _log_int(rng, 33, 2048)
    if rng.random() < 0.5:
        channels = (channels + 7) // 8 * 8
    time = 1 if op == "recurrence_step" else _log_int(rng, 1, 8192)
    most = {"recurrence_step": 16384 * 1152, "recurrence_forward": 512 * 128 * 1152,
            "recurrence_train": 512 * 128 * 1152}[op] // (2 if dtype == "f32" else 1)
    batch = _log_int(rng, 1, max(1, min(16384, most // (time * channels))))
    return _rec(None, op, batch, time, channels, dtype, rng.choice(["batch", "time"]), rng.random() < 0.5,
                rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------------

def _sequence(gen, case, scale=1.0, shift=0.0):
    """[batch, time, channels] in the case's type; a time-major case is a transposed view of the [time, batch,
    channels] array that a rollout leaves behind."""
    b, t, c = case["batch"], case["time"], case["channels"]
    shape = (t, b, c) if case["layout"] == "time" else (b, t, c)
    v = torch.randn(shape, generator=gen, device=DEVICE).mul_(scale).add_(shift).to(DTYPES[case["dtype"]])
    return v.transpose(0, 1) if case["layout"] == "time" else v


def _resets(gen, case):
    if not case["reset"]:
        return None
    b, t = case["batch"], case["time"]
    shape = (t, b) if case["layout"] == "time" else (b, t)
    r = (torch.rand(shape, generator=gen, device=DEVICE) < 0.01).to(torch.uint8)
    return r.transpose(0, 1) if case["layout"] == "time" else r


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"].startswith("norm"):
        n, w = case["rows"], case["width"]
        # a residual stream: a few units are much larger than the rest, and none is centred
        loud = torch.exp(0.5 * torch.randn((w,), generator=gen, device=DEVICE))
        shift = torch.randn((w,), generator=gen, device=DEVICE)
        s["x"] = (torch.randn((n, w), generator=gen, device=DEVICE) * loud + shift).to(dtype)
        s["residual"] = torch.randn((n, w), generator=gen, device=DEVICE).to(dtype) if case["residual"] else None
        s["w"] = 1.0 + 0.1 * torch.randn((w,), generator=gen, device=DEVICE)
        s["b"] = 0.1 * torch.randn((w,), generator=gen, device=DEVICE)
        if case["op"] == "norm_train":
            s["dy"] = torch.randn((n, w), generator=gen, device=DEVICE).to(dtype)
            s["dsum"] = torch.randn((n, w), generator=gen, device=DEVICE).to(dtype) if case["residual"] else None
        if own:
            from paper_2603_12145_b200 import layer_norm
            s["handle"] = layer_norm.LayerNorm(w, eps=EPS, dtype=dtype)
        return s
    if case["op"] == "orthogonal":
        b, m, n = case["batch"], case["rows"], case["cols"]
        # momentum: a few strong directions over a full-rank rest of the same size
        rank = max(1, min(m, n) // 16)
        size = torch.exp(-2.0 * torch.arange(rank, device=DEVICE) / rank)
        u = torch.randn((b, m, rank), generator=gen, device=DEVICE) * size
        v = torch.randn((b, rank, n), generator=gen, device=DEVICE)
        s["g"] = (1e-3 * (u @ v * (2.0 / rank) ** 0.5 + torch.randn((b, m, n), generator=gen, device=DEVICE))).to(dtype)
        if own:
            from paper_2603_12145_b200 import orthogonal
            s["handle"] = orthogonal.Orthogonal(m, n, dtype=dtype, steps=STEPS, coefficients=(NS_A, NS_B, NS_C), eps=NS_EPS)
        return s
    b, c = case["batch"], case["channels"]
    step = case["op"] == "recurrence_step"
    s["x"], s["r"], s["i"] = _sequence(gen, case), _sequence(gen, case, shift=1.0), _sequence(gen, case)
    s["reset"] = _resets(gen, case)
    # memories of a few to a thousand steps
    s["a"] = -torch.exp(torch.rand((c,), generator=gen, device=DEVICE) * math.log(500.0) + math.log(1e-3))
    s["state"] = None
    if step or case["carry"]:
        s["state"] = torch.randn((b, c), generator=gen, device=DEVICE)
    if case["op"] == "recurrence_train":
        s["dy"] = _sequence(gen, case)
        s["dstate_out"] = torch.randn((b, c), generator=gen, device=DEVICE) if case["carry"] else None
    if own:
        from paper_2603_12145_b200 import gated_recurrence
        s["handle"] = gated_recurrence.GatedRecurrence(c, dtype=dtype)
    if step:
        for key in ("x", "r", "i", "reset"):
            if s[key] is not None:
                s[key] = s[key][:, 0]
    return s


# ---- the package's kernels ------------------------------------------------------------

def _run_own(s):
    case, h, op = s["case"], s["handle"], s["case"]["op"]
    if op == "orthogonal":
        return {"update": h.update(s["g"])}
    if op.startswith("norm"):
        train = op == "norm_train"
        saved = h.saved(case["rows"]) if train else None
        if case["residual"]:
            y, total = h.forward(s["x"], s["w"], s["b"], residual=s["residual"], saved=saved)
            out = {"y": y, "sum": total}
        else:
            total = s["x"]
            out = {"y": h.forward(total, s["w"], s["b"], saved=saved)}
        if train:
            out["dx"], out["dw"], out["db"] = h.backward(s["dy"], total, s["w"], saved, dsum=s["dsum"])
        return out
    if op == "recurrence_step":
        state = torch.empty_like(s["state"])
        y = h.step(s["x"], s["r"], s["i"], s["a"], s["state"], done=s["reset"], state_out=state)
        return {"y": y, "state": state}
    state = h.state(case["batch"])
    train = op == "recurrence_train"
    saved = h.saved(case["batch"], case["time"]) if train else None
    y = h.sequence(s["x"], s["r"], s["i"], s["a"], reset=s["reset"], state=s["state"], state_out=state, saved=saved)
    out = {"y": y, "state": state}
    if train:
        grads = h.backward(s["dy"], s["x"], s["r"], s["i"], s["a"], saved, reset=s["reset"],
                           dstate_out=s["dstate_out"], want_dstate=s["state"] is not None)
        for key in ("dx", "dr", "di", "da", "dstate"):
            if grads[key] is not None:
                out[key] = grads[key]
    return out


# ---- plain forms: elementary operations in binary32 -----------------------------------

def _plain_norm(s):
    dtype = s["x"].dtype
    x = s["x"]
    out = {}
    if s["residual"] is not None:
        x = (x.float() + s["residual"].float()).to(dtype)      # the stream is of its type: what goes on is what is normalised
        out["sum"] = x
    x = x.float()
    centred = x - x.mean(dim=1, keepdim=True)
    scale = torch.rsqrt((centred * centred).mean(dim=1, keepdim=True) + EPS)
    z = centred * scale
    out["y"] = (z * s["w"] + s["b"]).to(dtype)
    if s["case"]["op"] == "norm_train":
        dy = s["dy"].float()
        c = dy * s["w"]
        dx = scale * (c - c.mean(dim=1, keepdim=True) - z * (c * z).mean(dim=1, keepdim=True))
        if s["dsum"] is not None:
            dx = dx + s["dsum"].float()
        out["dx"] = dx.to(dtype)
        out["dw"] = (dy * z).sum(dim=0)
        out["db"] = dy.sum(dim=0)
    return out


def _doubling(rate, v):
    """v_t + e^rate_t v_{t-1} + e^(rate_t + rate_{t-1}) v_{t-2} + ... along the first dimension.  The rates are added up:
    products of decays just below one gather their roundings over long sequences."""
    d, time = 1, v.shape[0]
    while d < time:
        v = torch.cat([v[:d], v[d:] + torch.exp(rate[d:]) * v[:-d]])
        rate = torch.cat([rate[:d], rate[d:] + rate[:-d]])
        d *= 2
    return v


def _plain_recurrence(s):
    case, dtype = s["case"], s["x"].dtype
    step = case["op"] == "recurrence_step"

    def seq(key):   # time first, binary32
        return (s[key].unsqueeze(0) if step else s[key].transpose(0, 1)).float()

    x, sr, si = seq("x"), torch.sigmoid(seq("r")), torch.sigmoid(seq("i"))
    rate = s["a"] * sr
    decay = torch.exp(rate)
    gain = torch.sqrt(-torch.expm1(2.0 * rate))
    kept, lasting = decay, rate
    if s["reset"] is not None:
        r = s["reset"].unsqueeze(0) if step else s["reset"].transpose(0, 1)
        kept = decay * (r == 0).float().unsqueeze(2)
        lasting = torch.where((r != 0).unsqueeze(2), float("-inf"), rate)
    u = si * x
    v = gain * u
    if s["state"] is not None:
        v = torch.cat([v[:1] + kept[:1] * s["state"], v[1:]])
    h = _doubling(lasting, v)
    back = (lambda t: t[0]) if step else (lambda t: t.transpose(0, 1))
    out = {"y": back(h).to(dtype), "state": h[-1].clone()}
    if case["op"] != "recurrence_train":
        return out
    g = seq("dy")
    if s["dstate_out"] is not None:
        g = torch.cat([g[:-1], g[-1:] + s["dstate_out"]])
    ahead = torch.cat([lasting[1:], torch.zeros_like(lasting[:1])]).flip(0)
    g = _doubling(ahead, g.flip(0)).flip(0)
    first = s["state"].unsqueeze(0) if s["state"] is not None else torch.zeros_like(h[:1])
    before = torch.cat([first, h[:-1]])
    drate = g * (kept * before - u * decay * decay / gain)
    out["dx"] = back(g * gain * si).to(dtype)
    out["di"] = back(g * gain * x * si * (1.0 - si)).to(dtype)
    out["dr"] = back(drate * rate * (1.0 - sr)).to(dtype)
    out["da"] = (drate * sr).sum(dim=(0, 1))
    if s["state"] is not None:
        out["dstate"] = kept[0] * g[0]
    return out


def _plain_orthogonal(s):
    x = s["g"].float()
    x = x / (torch.sqrt((x * x).sum(dim=(1, 2), keepdim=True)) + NS_EPS)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    for _ in range(STEPS):
        a = x @ x.transpose(1, 2)
        x = NS_A * x + (NS_B * a + NS_C * (a @ a)) @ x
    if tall:
        x = x.transpose(1, 2)
    return {"update": x.to(torch.bfloat16)}


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "orthogonal":
        return _plain_orthogonal(state)
    return _plain_norm(state) if op.startswith("norm") else _plain_recurrence(state)


# ---- the definitions in binary64 --------------------------------------------------------

def _exact_norm(case, s):
    out = {}
    x = s["x"].double()
    if case["residual"]:
        x = (x + s["residual"].double()).to(s["x"].dtype).double()
        out["sum"] = x
    mean = x.sum(dim=1) / case["width"]
    var = ((x - mean.unsqueeze(1)) ** 2).sum(dim=1) / case["width"]
    z = (x - mean.unsqueeze(1)) / torch.sqrt(var + EPS).unsqueeze(1)
    w = s["w"].double()
    out["y"] = z * w + s["b"].double()
    if case["op"] == "norm_train":
        dy = s["dy"].double()
        dz = dy * w
        along = (dz * z).sum(dim=1, keepdim=True) / case["width"]
        dx = (dz - dz.sum(dim=1, keepdim=True) / case["width"] - z * along) / torch.sqrt(var + EPS).unsqueeze(1)
        out["dx"] = dx if s["dsum"] is None else dx + s["dsum"].double()
        out["dw"] = torch.einsum("nw,nw->w", dy, z)
        out["db"] = dy.sum(dim=0)
    return out


def _exact_recurrence(case, s):
    step, train = case["op"] == "recurrence_step", case["op"] == "recurrence_train"
    at = (lambda key, t: s[key].double()) if step else (lambda key, t: s[key][:, t].double())
    batch, time, c = case["batch"], case["time"], case["channels"]
    a = s["a"].double()
    start = s["state"].double() if s["state"] is not None else torch.zeros((batch, c), dtype=torch.float64, device=a.device)

    def fresh(t):                                        # rows whose episode starts at t
        if s["reset"] is None:
            return torch.zeros((batch, 1), dtype=torch.bool, device=a.device)
        return (s["reset"] if step else s["reset"][:, t]).view(batch, 1) != 0

    y = torch.empty((batch, time, c), dtype=torch.float64, device=a.device)
    h = start
    for t in range(time):
        h = torch.where(fresh(t), torch.zeros_like(h), h)
        rate = a / (1 + torch.exp(-at("r", t)))
        h = torch.exp(rate) * h + torch.sqrt(-torch.expm1(2 * rate)) * at("x", t) / (1 + torch.exp(-at("i", t)))
        y[:, t] = h
    out = {"y": y[:, 0] if step else y, "state": h}
    if not train:
        return out
    dx, dr, di = torch.empty_like(y), torch.empty_like(y), torch.empty_like(y)
    da = torch.zeros_like(a)
    g = torch.zeros_like(h) if s["dstate_out"] is None else s["dstate_out"].double()
    for t in range(time - 1, -1, -1):
        g = g + at("dy", t)
        past = torch.where(fresh(t), torch.zeros_like(g), y[:, t - 1] if t > 0 else start)
        sr, si, x = torch.sigmoid(at("r", t)), torch.sigmoid(at("i", t)), at("x", t)
        decay, gain = torch.exp(a * sr), torch.sqrt(-torch.expm1(2 * a * sr))
        dgain, ddecay = g * si * x, g * past
        drate = ddecay * decay - dgain * decay ** 2 / gain
        dx[:, t], di[:, t] = g * gain * si, g * gain * x * si * (1 - si)
        dr[:, t] = drate * a * sr * (1 - sr)
        da += (drate * sr).sum(dim=0)
        g = torch.where(fresh(t), torch.zeros_like(g), g * decay)
    out.update(dx=dx, dr=dr, di=di, da=da)
    if s["state"] is not None:
        out["dstate"] = g
    return out


def _exact_orthogonal(s):
    found = []
    for g in s["g"].double():
        x = g / (torch.linalg.matrix_norm(g) + NS_EPS)
        for _ in range(STEPS):                           # the small side's product, whichever it is
            if x.shape[0] <= x.shape[1]:
                gram = x.mm(x.t())
                x = NS_A * x + NS_B * gram.mm(x) + NS_C * gram.mm(gram).mm(x)
            else:
                gram = x.t().mm(x)
                x = NS_A * x + NS_B * x.mm(gram) + NS_C * x.mm(gram.mm(gram))
        found.append(x)
    return {"update": torch.stack(found)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orthogonal":
        return _exact_orthogonal(s)
    return _exact_norm(case, s) if case["op"].startswith("norm") else _exact_recurrence(case, s)


# ---- what a pass cannot do without --------------------------------------------------------

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op.startswith("norm"):
        n, w = case["rows"], case["width"]
        streams = 4 if case["residual"] else 2                  # x, y; the residual and the sum
        moved, flops = streams * n * w * size + 8 * w, 9 * n * w
        if op == "norm_train":
            moved += (3 if case["residual"] else 2) * n * w * size + 8 * w      # dy, dx, the sum's gradient
            flops += 14 * n * w
        return {"bytes": moved, "flops": flops}
    if op == "orthogonal":
        b, m, n = case["batch"], case["rows"], case["cols"]
        k, l = min(m, n), max(m, n)
        # of the symmetric products one half
        return {"bytes": b * m * n * (size + 2), "flops": b * STEPS * (3 * k * k * l + k * k * k)}
    cells, c = case["batch"] * case["time"] * case["channels"], case["channels"]
    mask = case["batch"] * case["time"] if case["reset"] else 0
    state = 4 * case["batch"] * c
    moved, flops = 4 * cells * size + mask + 4 * c + state, 14 * cells
    if op == "recurrence_step" or case["carry"]:
        moved += state
    if op == "recurrence_train":
        moved += 4 * cells * size + 4 * c + (2 * state if case["carry"] else 0)
        flops += 30 * cells
    return {"bytes": moved, "flops": flops}
