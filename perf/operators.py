"""The cases on which the sequence-policy operators are measured: the short causal
convolution and the selective state space scan of ssm.py (whole sequences, their
gradients, single tokens) and the gated feed-forward block of gated_ffn.py (forward,
training step, few rows).

`run` computes a case with the package's kernels where `own` is true and otherwise from
elementary torch operations in binary32; `exact` evaluates the operators' definitions in
binary64, step by step.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DEVICE = "cuda"
GELU_C, GELU_K = math.sqrt(2.0 / math.pi), 0.044715


# ---- cases --------------------------------------------------------------------------

def _scan(name, kind, batch, time, channels, states=16, groups=1, dtype="bf16", layout="batch",
          reset=False, carry=False, gate=True):
    return {"name": name, "op": kind, "batch": batch, "time": time, "channels": channels, "states": states,
            "groups": groups, "dtype": dtype, "layout": layout, "reset": reset, "carry": carry, "gate": gate}


def _conv(name, kind, batch, time, channels, width=4, dtype="bf16", layout="batch", reset=False, carry=False):
    return {"name": name, "op": kind, "batch": batch, "time": time, "channels": channels, "width": width,
            "dtype": dtype, "layout": layout, "reset": reset, "carry": carry}


def _ffn(name, kind, rows, model, hidden, activation="silu", dtype="bf16"):
    return {"name": name, "op": kind, "rows": rows, "model": model, "hidden": hidden,
            "activation": activation, "dtype": dtype}


def listed():
    return [
        # one agent step of a few envs with a state-space policy twice as wide as the GRU policy's 576 units
        _scan("scan_step_64", "scan_step", 64, 1, 1152, reset=True),
        # one agent step of a large batch of envs: the recurrent state passes through memory once
        _scan("scan_step_16384", "scan_step", 16384, 1, 1152, reset=True),
        # one long prompt: a single row, whose time axis is all there is to split
        _scan("scan_prompt_1x8192", "scan_forward", 1, 8192, 2048),
        # training on a rollout as the env writes it: time-major, episodes end inside, state carried in
        _scan("scan_train_512x128", "scan_train", 512, 128, 1152, layout="time", reset=True, carry=True),
        # training in binary32 on odd sizes: states beyond one register block, channels in two groups
        _scan("scan_train_odd_f32", "scan_train", 3, 777, 330, states=24, groups=2, dtype="f32"),
        # the convolution's single-token form in front of the small agent step
        _conv("conv_step_64", "conv_step", 64, 1, 1152, reset=True),
        # the convolution over the rollout of the training case, with its gradients
        _conv("conv_train_1024x128", "conv_train", 1024, 128, 1152, layout="time", reset=True, carry=True),
        # a single token through a block of generic width: its weights have to be read once
        _ffn("ffn_token_1", "ffn_forward", 1, 2048, 8192),
        # the block in the policy loop at 64 envs
        _ffn("ffn_rows_64", "ffn_forward", 64, 576, 1536),
        # a ragged prompt, binary16, sizes that no tile divides
        _ffn("ffn_odd_f16", "ffn_forward", 1003, 1000, 2504, activation="gelu", dtype="f16"),
        # the policy's block on a rollout of 512 envs x 128 steps: many rows, small weights
        _ffn("ffn_train_65536", "ffn_train", 65536, 576, 1536),
        # training at generic width
        _ffn("ffn_train_8192", "ffn_train", 8192, 2048, 8192),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["scan_step", "scan_forward", "scan_train", "scan_train", "conv_step", "conv_train",
                     "ffn_forward", "ffn_forward", "ffn_train"])
    if op.startswith("ffn"):
        model, hidden = 8 * _log_int(rng, 8, 256), 8 * _log_int(rng, 8, 1024)
        most = 8192 * 2048 * 8192 if op == "ffn_train" else 1003 * 2048 * 8192
        rows = _log_int(rng, 1, max(1, min(65536, most // (model * hidden))))
        return _ffn(None, op, rows, model, hidden, rng.choice(["silu", "gelu"]), rng.choice(["bf16", "bf16", "f16"]))
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    layout = rng.choice(["batch", "time"])
    channels = _log_int(rng, 33, 2048)
    reset, carry = rng.random() < 0.5, rng.random() < 0.5
    if op.startswith("conv"):
        time = 1 if op == "conv_step" else _log_int(rng, 1, 8192)
        batch = _log_int(rng, 1, max(1, min(16384, 1024 * 128 * 1152 // (time * channels))))
        return _conv(None, op, batch, time, channels, rng.choice([2, 3, 4, 4]), dtype, layout, reset, carry)
    states = rng.choice([1, 4, 8, 16, 16, 16, 24, 32, 64])
    groups = rng.choice([1, 1, 2, 3])
    channels -= channels % groups
    time = 1 if op == "scan_step" else _log_int(rng, 1, 8192)
    most = {"scan_step": 16384 * 1152 * 16, "scan_forward": 8192 * 2048 * 16, "scan_train": 512 * 128 * 1152 * 16}[op]
    batch = _log_int(rng, 1, max(1, min(16384, most // (time * channels * states))))
    return _scan(None, op, batch, time, channels, states, groups, dtype, layout, reset, carry, rng.random() < 0.8)


# ---- inputs -------------------------------------------------------------------------

def _sequence(gen, case, features, scale=1.0):
    """[batch, time, features] in the case's type; a time-major case is a transposed view of
    the [time, batch, features] array that a rollout leaves behind."""
    b, t = case["batch"], case["time"]
    shape = (t, b, features) if case["layout"] == "time" else (b, t, features)
    v = (torch.randn(shape, generator=gen, device=DEVICE) * scale).to(DTYPES[case["dtype"]])
    return v.transpose(0, 1) if case["layout"] == "time" else v


def _resets(gen, case):
    b, t = case["batch"], case["time"]
    if not case["reset"]:
        return None
    shape = (t, b) if case["layout"] == "time" else (b, t)
    r = (torch.rand(shape, generator=gen, device=DEVICE) < 0.01).to(torch.uint8)
    return r.transpose(0, 1) if case["layout"] == "time" else r


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"].startswith("ffn"):
        n, m, h = case["rows"], case["model"], case["hidden"]
        s["x"] = torch.randn((n, m), generator=gen, device=DEVICE).to(dtype)
        s["w_in"] = (torch.randn((2 * h, m), generator=gen, device=DEVICE) * m ** -0.5).to(dtype)
        s["w_out"] = (torch.randn((m, h), generator=gen, device=DEVICE) * h ** -0.5).to(dtype)
        if case["op"] == "ffn_train":
            s["dy"] = torch.randn((n, m), generator=gen, device=DEVICE).to(dtype)
        if own:
            from paper_2603_12145_b200 import gated_ffn
            s["handle"] = gated_ffn.GatedFfn(m, h, activation=case["activation"], dtype=dtype)
        return s
    b, d = case["batch"], case["channels"]
    step = case["op"].endswith("step")
    s["x"] = _sequence(gen, case, d)
    s["reset"] = _resets(gen, case)
    if case["op"].startswith("conv"):
        w = case["width"]
        s["w"] = torch.randn((d, w), generator=gen, device=DEVICE) * w ** -0.5
        s["bias"] = torch.randn((d,), generator=gen, device=DEVICE) * 0.1
        s["history"] = None
        if step or case["carry"]:
            s["history"] = torch.randn((b, w - 1, d), generator=gen, device=DEVICE).to(dtype)
        if case["op"] == "conv_train":
            s["dy"] = _sequence(gen, case, d)
        if own:
            from paper_2603_12145_b200 import ssm
            s["handle"] = ssm.Ssm(d, states=16, groups=1, width=w, dtype=dtype)
    else:
        n, g = case["states"], case["groups"]
        s["dt"] = _sequence(gen, case, d, 0.5)
        s["b"] = _sequence(gen, case, g * n)
        s["c"] = _sequence(gen, case, g * n)
        s["z"] = _sequence(gen, case, d) if case["gate"] else None
        # decay rates spread over 1 .. states, steps of 0.001 .. 0.1 at dt = 0
        rate = torch.arange(1, n + 1, device=DEVICE, dtype=torch.float32)
        s["a"] = -rate * torch.exp(0.1 * torch.randn((d, n), generator=gen, device=DEVICE))
        s["d"] = 1.0 + 0.1 * torch.randn((d,), generator=gen, device=DEVICE)
        start = torch.exp(torch.rand((d,), generator=gen, device=DEVICE) * math.log(100.0) + math.log(1e-3))
        s["dt_bias"] = start + torch.log(-torch.expm1(-start))
        s["state"] = None
        if step or case["carry"]:
            s["state"] = 0.5 * torch.randn((b, d, n), generator=gen, device=DEVICE)
        if case["op"] == "scan_train":
            s["dy"] = _sequence(gen, case, d)
        if own:
            from paper_2603_12145_b200 import ssm
            s["handle"] = ssm.Ssm(d, states=n, groups=g, width=4, dtype=dtype)
    if step:
        for key in ("x", "dt", "z", "b", "c", "reset"):
            if s.get(key) is not None:
                s[key] = s[key][:, 0]
    return s


# ---- the package's kernels ------------------------------------------------------------

def _run_own(s):
    case, h = s["case"], s["handle"]
    op = case["op"]
    if op == "ffn_forward":
        return {"y": h.forward(s["x"], s["w_in"], s["w_out"])}
    if op == "ffn_train":
        saved = h.saved(case["rows"])
        y = h.forward(s["x"], s["w_in"], s["w_out"], saved=saved)
        dx, dw_in, dw_out = h.backward(s["dy"], s["x"], s["w_in"], s["w_out"], saved)
        return {"y": y, "dx": dx, "dw_in": dw_in, "dw_out": dw_out}
    if op == "conv_step":
        history = torch.empty_like(s["history"])
        y = h.conv_step(s["x"], s["history"], s["w"], s["bias"], done=s["reset"], history_out=history)
        return {"y": y, "history": history}
    if op == "conv_train":
        history = h.history(case["batch"])
        y = h.conv(s["x"], s["w"], s["bias"], reset=s["reset"], history=s["history"], history_out=history)
        dx, dw, dbias = h.conv_backward(s["dy"], s["x"], s["w"], s["bias"], reset=s["reset"], history=s["history"])
        return {"y": y, "history": history, "dx": dx, "dw": dw, "dbias": dbias}
    if op == "scan_step":
        state = torch.empty_like(s["state"])
        y = h.scan_step(s["x"], s["dt"], s["a"], s["b"], s["c"], s["state"], d=s["d"], z=s["z"],
                        dt_bias=s["dt_bias"], done=s["reset"], state_out=state)
        return {"y": y, "state": state}
    state = h.state(case["batch"])
    if op == "scan_forward":
        y = h.scan(s["x"], s["dt"], s["a"], s["b"], s["c"], d=s["d"], z=s["z"], dt_bias=s["dt_bias"],
                   reset=s["reset"], state=s["state"], state_out=state)
        return {"y": y, "state": state}
    saved = h.saved(case["batch"], case["time"])
    y = h.scan(s["x"], s["dt"], s["a"], s["b"], s["c"], d=s["d"], z=s["z"], dt_bias=s["dt_bias"],
               reset=s["reset"], state=s["state"], state_out=state, saved=saved)
    grads = h.scan_backward(s["dy"], s["x"], s["dt"], s["a"], s["b"], s["c"], saved, d=s["d"], z=s["z"],
                            dt_bias=s["dt_bias"], reset=s["reset"], want_dstate=s["state"] is not None)
    out = {"y": y, "state": state}
    for key in ("dx", "ddt", "da", "db", "dc", "dd", "dz", "ddt_bias", "dstate"):
        if grads[key] is not None:
            out[key] = grads[key]
    return out


# ---- plain forms: elementary operations in binary32 -----------------------------------

def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _softplus(v):
    return torch.clamp(v, min=0.0) + torch.log1p(torch.exp(-torch.abs(v)))


def _act(v, name):
    if name == "silu":
        return v * _sigmoid(v)
    return 0.5 * v * (1.0 + torch.tanh(GELU_C * (v + GELU_K * v * v * v)))


def _dact(v, name):
    if name == "silu":
        g = _sigmoid(v)
        return g * (1.0 + v * (1.0 - g))
    th = torch.tanh(GELU_C * (v + GELU_K * v * v * v))
    return 0.5 * (1.0 + th) + 0.5 * v * (1.0 - th * th) * GELU_C * (1.0 + 3.0 * GELU_K * v * v)


def _plain_ffn(s):
    case, dtype = s["case"], s["x"].dtype
    hid, act = case["hidden"], case["activation"]
    x, w_in, w_out = s["x"].float(), s["w_in"].float(), s["w_out"].float()
    pre = x @ w_in.t()
    gate, up = pre[:, :hid], pre[:, hid:]
    a = _act(gate, act)
    h = a * up
    out = {"y": (h @ w_out.t()).to(dtype)}
    if case["op"] == "ffn_train":
        dy = s["dy"].float()
        dh = dy @ w_out
        dpre = torch.cat([dh * up * _dact(gate, act), dh * a], dim=1)
        out["dx"] = (dpre @ w_in).to(dtype)
        out["dw_in"] = (dpre.t() @ x).to(dtype)
        out["dw_out"] = (dy.t() @ h).to(dtype)
    return out


def _plain_conv(s):
    case, dtype = s["case"], s["x"].dtype
    w, width = s["w"], case["width"]
    step = case["op"] == "conv_step"
    x = (s["x"].unsqueeze(1) if step else s["x"]).float()
    batch, time, d = x.shape
    reset = s["reset"]
    if reset is not None and step:
        reset = reset.unsqueeze(1)
    past = s["history"].float() if s["history"] is not None else x.new_zeros((batch, width - 1, d))
    ext = torch.cat([past, x], dim=1)
    # a tap is dropped where an episode starts between it and t
    keep = [None] * width
    if reset is not None:
        start = torch.cumsum(reset.to(torch.int32), dim=1)
        start = torch.cat([start.new_zeros((batch, width - 1)), start], dim=1)
        for k in range(width):
            keep[k] = (start[:, k:k + time] == start[:, width - 1:]).float().unsqueeze(2)
    pre = s["bias"].expand(batch, time, d)
    for k in range(width):
        tap = ext[:, k:k + time]
        pre = pre + (tap if keep[k] is None else tap * keep[k]) * w[:, k]
    out = {"y": _act(pre, "silu").to(dtype)}
    tail = ext[:, time:]
    if reset is not None:
        tail = torch.where((start[:, time:] == start[:, -1:]).unsqueeze(2), tail, torch.zeros_like(tail))
    out["history"] = tail.to(dtype)
    if step:
        out["y"] = out["y"][:, 0]
        return out
    dpre = s["dy"].float() * _dact(pre, "silu")
    dext = torch.zeros_like(ext)
    dw = []
    for k in range(width):
        tap = ext[:, k:k + time]
        dk = dpre if keep[k] is None else dpre * keep[k]
        dext[:, k:k + time] += dk * w[:, k]
        dw.append((dk * tap).sum(dim=(0, 1)))
    out["dx"] = dext[:, width - 1:].to(dtype)
    out["dw"] = torch.stack(dw, dim=1)
    out["dbias"] = dpre.sum(dim=(0, 1))
    return out


def _plain_scan(s):
    case, dtype = s["case"], s["x"].dtype
    step = case["op"] == "scan_step"
    g, n = case["groups"], case["states"]

    def seq(key):   # time first, binary32
        v = s.get(key)
        if v is None:
            return None
        return (v.unsqueeze(0) if step else v.transpose(0, 1)).float()

    x, raw, z = seq("x"), seq("dt"), seq("z")
    time, batch, d = x.shape
    raw = raw + s["dt_bias"]
    delta = _softplus(raw)

    def grouped(v):
        return v.reshape(v.shape[:-1] + (g, d // g, 1))

    xg, dg = grouped(x), grouped(delta)
    bg = seq("b").reshape(time, batch, g, 1, n)
    cg = seq("c").reshape(time, batch, g, 1, n)
    a = s["a"].reshape(g, d // g, n)
    decay = torch.exp(dg * a)
    if s["reset"] is not None:
        r = s["reset"].unsqueeze(0) if step else s["reset"].transpose(0, 1)
        decay = decay * (r == 0).float().reshape(time, batch, 1, 1, 1)
    h0 = s["state"]
    h = h0.reshape(batch, g, d // g, n) if h0 is not None else x.new_zeros((batch, g, d // g, n))
    first = h
    hs = (dg * xg) * bg
    for t in range(time):
        h = torch.addcmul(hs[t], decay[t], h)
        hs[t] = h
    ypre = (hs * cg).sum(dim=-1).reshape(time, batch, d) + s["d"] * x
    y = ypre if z is None else ypre * _act(z, "silu")
    back = (lambda v: v[0]) if step else (lambda v: v.transpose(0, 1))
    out = {"y": back(y).to(dtype), "state": hs[time - 1].reshape(batch, d, n).clone()}
    if case["op"] != "scan_train":
        return out
    dy = seq("dy")
    grad = dy if z is None else dy * _act(z, "silu")
    if z is not None:
        out["dz"] = back(dy * ypre * _dact(z, "silu")).to(dtype)
    gg = grouped(grad)
    dh = gg * cg
    for t in range(time - 2, -1, -1):
        dh[t].addcmul_(decay[t + 1], dh[t + 1])
    if h0 is not None:
        out["dstate"] = (decay[0] * dh[0]).reshape(batch, d, n)
    out["dc"] = back((gg * hs).sum(dim=3).reshape(time, batch, g * n)).to(dtype)
    hs = torch.cat([first.unsqueeze(0), hs[:-1]])          # the state before each step
    decay.mul_(hs)
    del hs
    db = (dh * (dg * xg)).sum(dim=3)
    out["db"] = back(db.reshape(time, batch, g * n)).to(dtype)
    dhb = (dh * bg).sum(dim=-1).reshape(time, batch, d)
    decay.mul_(dh)
    out["da"] = (decay * dg).sum(dim=(0, 1)).reshape(d, n)
    ddelta = (decay * a).sum(dim=-1).reshape(time, batch, d) + x * dhb
    out["dx"] = back(s["d"] * grad + delta * dhb).to(dtype)
    ddt = ddelta * _sigmoid(raw)
    out["ddt"] = back(ddt).to(dtype)
    out["ddt_bias"] = ddt.sum(dim=(0, 1))
    out["dd"] = (grad * x).sum(dim=(0, 1))
    return out


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op.startswith("ffn"):
        return _plain_ffn(state)
    return _plain_conv(state) if op.startswith("conv") else _plain_scan(state)


# ---- the definitions in binary64 --------------------------------------------------------

def _exact_ffn(case, s):
    x, w_in, w_out = s["x"].double(), s["w_in"].double(), s["w_out"].double()
    n = case["hidden"]
    gate, up = x @ w_in[:n].t(), x @ w_in[n:].t()
    if case["activation"] == "silu":
        sg = torch.sigmoid(gate)
        act, slope = gate * sg, sg + gate * sg * (1 - sg)
    else:
        u = GELU_C * (gate + GELU_K * gate ** 3)
        act = 0.5 * gate * (1 + torch.tanh(u))
        slope = 0.5 * (1 + torch.tanh(u)) + 0.5 * gate / torch.cosh(u) ** 2 * GELU_C * (1 + 3 * GELU_K * gate ** 2)
    out = {"y": (act * up) @ w_out.t()}
    if case["op"] == "ffn_train":
        dy = s["dy"].double()
        dh = dy @ w_out
        dgate, dup = dh * up * slope, dh * act
        out["dx"] = dgate @ w_in[:n] + dup @ w_in[n:]
        out["dw_in"] = torch.cat([dgate.t() @ x, dup.t() @ x])
        out["dw_out"] = dy.t() @ (act * up)
    return out


def _exact_conv(case, s):
    step = case["op"] == "conv_step"
    x = s["x"].double()
    if step:
        x = x.unsqueeze(1)
    batch, time, d = x.shape
    width, w, bias = case["width"], s["w"].double(), s["bias"].double()
    reset = s["reset"]
    if reset is not None:
        reset = (reset.unsqueeze(1) if step else reset) != 0
    window = (s["history"].double() if s["history"] is not None else
              torch.zeros((batch, width - 1, d), dtype=torch.float64, device=x.device))
    train = case["op"] == "conv_train"
    y = torch.empty_like(x)
    age = torch.full((batch,), width, device=x.device)       # steps since the episode began, capped
    dx = torch.zeros_like(x)
    dw, dbias = torch.zeros_like(w), torch.zeros_like(bias)
    for t in range(time):
        age = age + 1
        if reset is not None:
            age = torch.where(reset[:, t], torch.zeros_like(age), age)
            window = torch.where(reset[:, t].view(batch, 1, 1), torch.zeros_like(window), window)
        taps = torch.cat([window, x[:, t:t + 1]], dim=1)
        pre = bias + (taps * w.t()).sum(dim=1)
        sg = torch.sigmoid(pre)
        y[:, t] = pre * sg
        if train:
            dpre = s["dy"][:, t].double() * (sg + pre * sg * (1 - sg))
            dbias += dpre.sum(dim=0)
            dw += (taps * dpre.unsqueeze(1)).sum(dim=0).t()
            for back in range(min(width, t + 1)):
                seen = (age >= back).view(batch, 1)
                dx[:, t - back] += torch.where(seen, dpre * w[:, width - 1 - back], torch.zeros_like(dpre))
        window = taps[:, 1:]
    out = {"y": y[:, 0] if step else y, "history": window}
    if train:
        out.update(dx=dx, dw=dw, dbias=dbias)
    return out


def _exact_scan(case, s):
    step, train = case["op"] == "scan_step", case["op"] == "scan_train"
    g, n = case["groups"], case["states"]
    names = ("x", "dt", "z", "b", "c", "dy", "reset")
    v = {k: None if s.get(k) is None else (s[k].unsqueeze(1) if step else s[k]) for k in names}
    batch, time, d = v["x"].shape
    a, dskip, dt_bias = s["a"].double(), s["d"].double(), s["dt_bias"].double()
    owner = torch.arange(d, device=a.device) // (d // g)      # a channel's group

    def at(key, t):
        return v[key][:, t].double()

    def shared(key, t):                                       # [batch, channels, states]
        return at(key, t).view(batch, g, n)[:, owner]

    h = (s["state"].double() if s["state"] is not None else
         torch.zeros((batch, d, n), dtype=torch.float64, device=a.device))
    y = torch.empty((batch, time, d), dtype=torch.float64, device=a.device)
    before = torch.empty((time if train else 0, batch, d, n), dtype=torch.float64, device=a.device)
    for t in range(time):
        if v["reset"] is not None:
            h = torch.where((v["reset"][:, t] != 0).view(batch, 1, 1), torch.zeros_like(h), h)
        if train:
            before[t] = h
        delta = torch.logaddexp(at("dt", t) + dt_bias, torch.zeros_like(dt_bias))
        h = torch.exp(delta.unsqueeze(2) * a) * h + (delta * at("x", t)).unsqueeze(2) * shared("b", t)
        out_t = (shared("c", t) * h).sum(dim=2) + dskip * at("x", t)
        y[:, t] = out_t if v["z"] is None else out_t * at("z", t) * torch.sigmoid(at("z", t))
    out = {"y": y[:, 0] if step else y, "state": h}
    if not train:
        return out
    grad = {k: torch.empty_like(y) for k in ("dx", "ddt", "dz")}
    db = torch.empty((batch, time, g * n), dtype=torch.float64, device=a.device)
    dc = torch.empty_like(db)
    da, dd, ddt_bias = torch.zeros_like(a), torch.zeros_like(dskip), torch.zeros_like(dskip)
    carry = torch.zeros_like(h)
    for t in range(time - 1, -1, -1):
        raw, x, z = at("dt", t) + dt_bias, at("x", t), None
        delta = torch.logaddexp(raw, torch.zeros_like(raw))
        decay = torch.exp(delta.unsqueeze(2) * a)
        h = decay * before[t] + (delta * x).unsqueeze(2) * shared("b", t)
        dy = at("dy", t)
        if v["z"] is not None:
            z = at("z", t)
            sg = torch.sigmoid(z)
            out_t = (shared("c", t) * h).sum(dim=2) + dskip * x
            grad["dz"][:, t] = dy * out_t * (sg + z * sg * (1 - sg))
            dy = dy * z * sg
        carry = carry + dy.unsqueeze(2) * shared("c", t)
        dc[:, t] = (dy.unsqueeze(2) * h).view(batch, g, d // g, n).sum(dim=2).reshape(batch, g * n)
        db[:, t] = (carry * (delta * x).unsqueeze(2)).view(batch, g, d // g, n).sum(dim=2).reshape(batch, g * n)
        into = carry * decay * before[t]
        da += (into * delta.unsqueeze(2)).sum(dim=0)
        pull = (carry * shared("b", t)).sum(dim=2)
        grad["dx"][:, t] = dskip * dy + delta * pull
        ddt = ((into * a).sum(dim=2) + x * pull) * torch.sigmoid(raw)
        grad["ddt"][:, t] = ddt
        ddt_bias += ddt.sum(dim=0)
        dd += (dy * x).sum(dim=0)
        carry = carry * decay
        if v["reset"] is not None:
            carry = torch.where((v["reset"][:, t] != 0).view(batch, 1, 1), torch.zeros_like(carry), carry)
    out.update(dx=grad["dx"], ddt=grad["ddt"], da=da, db=db, dc=dc, dd=dd, ddt_bias=ddt_bias)
    if v["z"] is not None:
        out["dz"] = grad["dz"]
    if s["state"] is not None:
        out["dstate"] = carry
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("ffn"):
        out = _exact_ffn(case, s)
    else:
        out = _exact_conv(case, s) if case["op"].startswith("conv") else _exact_scan(case, s)
    order = ("y", "history", "state", "dx", "ddt", "da", "db", "dc", "dd", "dz", "ddt_bias", "dstate",
             "dw", "dbias", "dw_in", "dw_out")
    return {k: out[k] for k in order if k in out}


# ---- what a pass cannot do without --------------------------------------------------------

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op.startswith("ffn"):
        n, m, h = case["rows"], case["model"], case["hidden"]
        moved = size * (2 * n * m + 3 * h * m)
        if op == "ffn_train":
            moved += size * (2 * n * m + 3 * h * m)
        return {"bytes": moved, "flops": (18 if op == "ffn_train" else 6) * n * m * h}
    rows, d = case["batch"] * case["time"], case["channels"]
    mask = rows if case["reset"] else 0
    if op.startswith("conv"):
        w = case["width"]
        past = case["batch"] * (w - 1) * d * size
        moved = 2 * rows * d * size + mask + 4 * d * (w + 1) + past
        flops = rows * d * (2 * w + 5)
        if op == "conv_step" or case["carry"]:
            moved += past
        if op == "conv_train":
            moved += 2 * rows * d * size + 4 * d * (w + 1)
            flops += rows * d * (4 * w + 8)
        return {"bytes": moved, "flops": flops}
    n, g = case["states"], case["groups"]
    state = 4 * case["batch"] * d * n
    wide, narrow = rows * d * size, rows * g * n * size
    streams = 4 if case["gate"] else 3                       # x, dt, (z) and y
    moved = streams * wide + 2 * narrow + mask + 4 * d * (n + 2) + state
    flops = rows * d * (7 * n + 16)
    if op == "scan_step" or case["carry"]:
        moved += state
    if op == "scan_train":
        moved += streams * wide + 2 * narrow + 4 * d * (n + 2) + (state if case["carry"] else 0)
        flops += rows * d * (14 * n + 24)
    return {"bytes": moved, "flops": flops}
