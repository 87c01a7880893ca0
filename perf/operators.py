"""The operators of a space-time network and its optimiser, as cases to be measured.

A network that marches a field along an axis of the grid mixes each row of nodes with a short causal
convolution and a selective state space scan; its weight matrices are updated with orthogonalised
momentum.  Each case is one call, or one forward and backward pair of calls, of those operators:

    conv_train   causal convolution with SiLU, forward and gradients
    conv_prompt  causal convolution with SiLU, forward with the window left for the next node
    scan_prompt  selective scan, forward with the state left for the next node
    scan_train   selective scan, forward and gradients
    step         one node for each row: convolution window and scan state moved on by one
    ortho        Newton-Schulz orthogonalisation of a stack of matrices
    muon         the optimiser's whole update of a stack of matrices

`own = False` computes the plain form in 32 bits with elementary torch operations, `own = True` calls
this package.  `exact` restates each operator in 64 bits, one node after the other.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NS_A, NS_B, NS_C = 3.4445, -4.775, 2.0315      # quintic of the Newton-Schulz iteration
EPS = 1e-7
LR, MU, WD = 0.02, 0.95, 0.01                  # optimiser settings of the muon cases


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a small network's training step on a 1000-node axis; a channel count that is no multiple of 4
        {"name": "conv_train_f32_odd", "op": "conv_train", "type": "f32", "batch": 4, "length": 1000, "channels": 333, "width": 4},
        # training of a wide network on long rows: as much as memory can move
        {"name": "conv_train_bf16_wide", "op": "conv_train", "type": "bf16", "batch": 8, "length": 8192, "channels": 2048, "width": 4},
        # inference of a small network on one row of 100 time nodes: latency
        {"name": "scan_prompt_f32_short", "op": "scan_prompt", "type": "f32", "batch": 1, "length": 100, "channels": 128, "states": 16},
        # one long row: few channels' rows for the whole GPU, so the axis has to be split
        {"name": "scan_prompt_bf16_long", "op": "scan_prompt", "type": "bf16", "batch": 1, "length": 16384, "channels": 1536, "states": 16},
        # many rows of a wide network: the throughput case
        {"name": "scan_prompt_bf16_wide", "op": "scan_prompt", "type": "bf16", "batch": 8, "length": 2048, "channels": 4096, "states": 16},
        # a training step on a 256 x 128 space-time grid, one row of 128 time nodes for each x
        {"name": "scan_train_f32_grid", "op": "scan_train", "type": "f32", "batch": 256, "length": 128, "channels": 64, "states": 16},
        # a training step of a wide network on long rows
        {"name": "scan_train_bf16_wide", "op": "scan_train", "type": "bf16", "batch": 4, "length": 4096, "channels": 2048, "states": 16},
        # marching one row by one node: latency
        {"name": "step_f32_one", "op": "step", "type": "f32", "batch": 1, "channels": 512, "states": 16, "width": 4},
        # marching all rows of a 256-node axis by one node: the states' traffic
        {"name": "step_bf16_rows", "op": "step", "type": "bf16", "batch": 256, "channels": 4096, "states": 16, "width": 4},
        # the hidden layers of a small network as one stack: latency
        {"name": "ortho_f32_layers", "op": "ortho", "type": "f32", "count": 8, "rows": 128, "cols": 128, "steps": 5},
        # the update of four odd-sized layers, taller than wide
        {"name": "muon_f32_odd", "op": "muon", "type": "f32", "count": 4, "rows": 1000, "cols": 333, "steps": 5},
        # the projection of a wide network
        {"name": "ortho_bf16_wide", "op": "ortho", "type": "bf16", "count": 1, "rows": 4096, "cols": 4096, "steps": 5},
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("conv_train", "conv_prompt", "scan_prompt", "scan_train", "step", "ortho", "muon"))
    case = {"op": op, "type": rng.choice(("f32", "bf16"))}
    if op in ("conv_train", "conv_prompt"):
        channels = _between(rng, 16, 4096)
        length = _between(rng, 1, 16384)
        most = max(1, min(256, (1 << 26) // (channels * length)))
        case |= {"batch": _between(rng, 1, most), "length": length, "channels": channels, "width": rng.choice((2, 3, 4))}
    elif op in ("scan_prompt", "scan_train"):
        channels = _between(rng, 16, 4096)
        states = rng.choice((4, 8, 16, 16, 24, 32))
        room = (1 << (30 if op == "scan_prompt" else 28)) // (channels * states)
        length = _between(rng, 1, min(16384, room))
        case |= {"batch": _between(rng, 1, max(1, min(256, room // length))), "length": length, "channels": channels, "states": states}
    elif op == "step":
        case |= {"batch": _between(rng, 1, 256), "channels": _between(rng, 16, 4096), "states": rng.choice((4, 8, 16, 16, 24, 32)), "width": rng.choice((2, 3, 4))}
    else:
        most = 1024 if case["type"] == "f32" else 4096
        rows = _between(rng, 16, most)
        cols = _between(rng, 16, most)
        room = max(1, min(32, (1 << 34) // (min(rows, cols) * rows * cols)))
        case |= {"count": _between(rng, 1, room), "rows": rows, "cols": cols, "steps": 5}
    return case


# ----------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    dt = TYPES[case["type"]]
    op = case["op"]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE) * scale

    def uniform(lo, hi, *shape):
        return torch.rand(*shape, generator=g, device=DEVICE) * (hi - lo) + lo

    s = {"op": op, "dtype": dt}
    if op in ("ortho", "muon"):
        # a gradient: products of activations and sensitivities, with a decaying spectrum, and noise
        k, m, n = case["count"], case["rows"], case["cols"]
        r = min(m, n) // 2 + 1
        decay = torch.arange(1, r + 1, device=DEVICE, dtype=torch.float32).pow(-0.5)
        grad = torch.bmm(normal(k, m, r) * decay, normal(k, r, n)) + 0.2 * normal(k, m, n)
        s |= {"grad": (grad * 1e-3).to(dt), "steps": case["steps"]}
        if op == "muon":
            s |= {"weight": normal(k, m, n, scale=0.05).to(dt), "momentum": normal(k, m, n, scale=3e-3)}
        return s
    b, c = case["batch"], case["channels"]
    if op != "step":
        length = case["length"]
    if "width" in case:
        w = case["width"]
        s |= {"weight": uniform(-0.5, 0.5, c, w), "bias": uniform(-0.5, 0.5, c)}
    if op in ("conv_train", "conv_prompt"):
        s |= {"x": normal(b, length, 2 * c).to(dt)[..., :c]}      # half of the input projection's output
        s |= {"window": normal(b, w - 1, c).to(dt)}
        if op == "conv_train":
            s |= {"gy": normal(b, length, c).to(dt)}
        return s
    n = case["states"]
    rank = max(1, c // 16)
    s |= {
        "A": -torch.arange(1, n + 1, device=DEVICE, dtype=torch.float32).repeat(c, 1) * uniform(0.8, 1.2, c, n),
        "D": uniform(0.5, 1.5, c),
        "delta_bias": torch.log(torch.expm1(torch.exp(uniform(math.log(1e-3), math.log(0.1), c)))),
    }
    lead = (b,) if op == "step" else (b, length)
    s |= {"z": normal(*lead, 2 * c).to(dt)[..., c:], "delta": normal(*lead, c, scale=0.5).to(dt)}
    bc = normal(*lead, rank + 2 * n).to(dt)                       # the projection that also gives delta
    s |= {"B": bc[..., rank:rank + n], "C": bc[..., rank + n:]}
    s |= {"state": normal(b, c, n, scale=0.1)}
    if op == "step":
        s |= {"x": normal(b, 2 * c).to(dt)[..., :c], "window": normal(b, w - 1, c).to(dt)}
    else:
        s |= {"u": normal(b, length, c).to(dt)}
        if op == "scan_train":
            s |= {"gout": normal(b, length, c).to(dt)}
    return s


# ------------------------------------------------------------------------------------ plain forms
def _silu(v):
    return v / (1 + torch.exp(-v))


def _silu_slope(v):
    g = 1 / (1 + torch.exp(-v))
    return g * (1 + v * (1 - g))


def _softplus(v):
    return torch.where(v > 20, v, torch.log1p(torch.exp(torch.clamp(v, max=20))))


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along axis 1 (h_{-1} = 0), in log2(length) doublings."""
    length, k = a.shape[1], 1
    a, b = a.clone(), b.clone()
    while k < length:
        b[:, k:] = b[:, k:] + a[:, k:] * b[:, :-k]
        a[:, k:] = a[:, k:] * a[:, :-k]
        k *= 2
    return b


def _plain_conv(s):
    f = torch.float32
    x, win, wt, bias = s["x"].to(f), s["window"].to(f), s["weight"], s["bias"]
    full = torch.cat((win, x), 1)
    taps = full.unfold(1, wt.shape[1], 1)                         # (batch, length, channels, width)
    pre = (taps * wt).sum(-1) + bias
    y = _silu(pre).to(s["dtype"])
    keep = full[:, full.shape[1] - wt.shape[1] + 1:].to(s["dtype"])
    if s["op"] == "conv_prompt":
        return {"y": y, "window": keep}
    g = s["gy"].to(f) * _silu_slope(pre)
    w = wt.shape[1]
    zeros = g.new_zeros(g.shape[0], w - 1, g.shape[2])
    gfull = (torch.cat((zeros, g, zeros), 1).unfold(1, w, 1) * wt.flip(1)).sum(-1)
    return {"y": y, "gx": gfull[:, w - 1:].to(s["dtype"]), "gwindow": gfull[:, :w - 1].to(s["dtype"]),
            "gweight": (taps * g.unsqueeze(-1)).sum((0, 1)), "gbias": g.sum((0, 1))}


def _plain_scan(s):
    f, dt = torch.float32, s["dtype"]
    u, raw, z = s["u"].to(f), s["delta"].to(f) + s["delta_bias"], s["z"].to(f)
    bt, ct, A, D = s["B"].to(f), s["C"].to(f), s["A"], s["D"]
    step = _softplus(raw)
    a = torch.exp(step.unsqueeze(-1) * A)
    b = (step * u).unsqueeze(-1) * bt.unsqueeze(2)
    b[:, 0] += a[:, 0] * s["state"]
    h = _scan(a, b)
    y = (h * ct.unsqueeze(2)).sum(-1) + D * u
    out, last = (y * _silu(z)).to(dt), h[:, -1].clone()
    if s["op"] == "scan_prompt":
        return {"out": out, "state": last}
    del b
    go = s["gout"].to(f)
    gy, gz = go * _silu(z), go * y * _silu_slope(z)
    gc = (h * gy.unsqueeze(-1)).sum(2)
    ah = a * torch.cat((s["state"].unsqueeze(1), h[:, :-1]), 1)   # what the step kept of the state before it
    del h
    nxt = torch.cat((a[:, 1:], torch.zeros_like(a[:, :1])), 1)
    adj = _scan(nxt.flip(1), (gy.unsqueeze(-1) * ct.unsqueeze(2)).flip(1)).flip(1)
    del nxt
    gb = (adj * (step * u).unsqueeze(-1)).sum(2)
    from_b = (adj * bt.unsqueeze(2)).sum(-1)
    gstate = a[:, 0] * adj[:, 0]
    ah *= adj
    gstep = (ah * A).sum(-1) + from_b * u
    graw = gstep / (1 + torch.exp(-raw))
    return {"out": out, "state": last, "gu": (step * from_b + D * gy).to(dt), "gdelta": graw.to(dt), "gz": gz.to(dt),
            "gB": gb.to(dt), "gC": gc.to(dt), "gA": (ah * step.unsqueeze(-1)).sum((0, 1)), "gD": (gy * u).sum((0, 1)),
            "gdelta_bias": graw.sum((0, 1)), "gstate": gstate}


def _plain_step(s):
    f, dt = torch.float32, s["dtype"]
    full = torch.cat((s["window"], s["x"].unsqueeze(1)), 1)
    u = _silu((full.to(f) * s["weight"].t()).sum(1) + s["bias"]).to(dt)
    s["window"].copy_(full[:, 1:])
    step = _softplus(s["delta"].to(f) + s["delta_bias"])
    v, z = u.to(f), s["z"].to(f)
    h = torch.exp(step.unsqueeze(-1) * s["A"]) * s["state"] + (step * v).unsqueeze(-1) * s["B"].to(f).unsqueeze(1)
    s["state"].copy_(h)
    out = ((h * s["C"].to(f).unsqueeze(1)).sum(-1) + s["D"] * v) * _silu(z)
    return {"u": u, "out": out.to(dt), "window": s["window"], "state": s["state"]}


def _newton_schulz(x, steps):
    turned = x.shape[1] > x.shape[2]
    if turned:
        x = x.transpose(1, 2)
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(steps):
        gram = torch.bmm(x.transpose(1, 2), x)
        x = NS_A * x + torch.bmm(x, NS_B * gram + NS_C * torch.bmm(gram, gram))
    return x.transpose(1, 2) if turned else x


def _plain_muon(s):
    grad = s["grad"].to(torch.float32)
    if s["op"] == "ortho":
        return {"out": _newton_schulz(grad, s["steps"]).to(s["dtype"])}
    s["momentum"].mul_(MU).add_(grad)
    update = _newton_schulz(grad + MU * s["momentum"], s["steps"])
    rate = LR * math.sqrt(max(1.0, grad.shape[1] / grad.shape[2]))
    s["weight"].copy_(((1 - LR * WD) * s["weight"].to(torch.float32) - rate * update).to(s["dtype"]))
    return {"weight": s["weight"], "momentum": s["momentum"]}


# --------------------------------------------------------------------------------- the package's
def _own(s):
    from paper_2607_18020_b200 import optim, sequence
    op = s["op"]
    if op in ("conv_train", "conv_prompt"):
        y, window = sequence.causal_conv_fwd(s["x"], s["weight"], s["bias"], state=s["window"], silu=True)
        if op == "conv_prompt":
            return {"y": y, "window": window}
        g = sequence.causal_conv_bwd(s["gy"], s["x"], s["weight"], s["bias"], state=s["window"], silu=True)
        return {"y": y, "gx": g.x, "gwindow": g.state, "gweight": g.weight, "gbias": g.bias}
    if op in ("scan_prompt", "scan_train"):
        args = (s["u"], s["delta"], s["A"], s["B"], s["C"])
        more = {"D": s["D"], "z": s["z"], "delta_bias": s["delta_bias"], "delta_softplus": True, "state": s["state"]}
        out, last, kept = sequence.selective_scan_fwd(*args, **more, keep=op == "scan_train")
        if op == "scan_prompt":
            return {"out": out, "state": last}
        g = sequence.selective_scan_bwd(s["gout"], *args, **more, kept=kept)
        return {"out": out, "state": last, "gu": g.u, "gdelta": g.delta, "gz": g.z, "gB": g.B, "gC": g.C, "gA": g.A, "gD": g.D,
                "gdelta_bias": g.delta_bias, "gstate": g.state}
    if op == "step":
        u = sequence.causal_conv_step(s["x"], s["window"], s["weight"], s["bias"], silu=True)
        out = sequence.selective_scan_step(s["state"], u, s["delta"], s["A"], s["B"], s["C"], D=s["D"], z=s["z"],
                                           delta_bias=s["delta_bias"], delta_softplus=True)
        return {"u": u, "out": out, "window": s["window"], "state": s["state"]}
    if op == "ortho":
        return {"out": optim.orthogonalize(s["grad"], steps=s["steps"], eps=EPS)}
    optim.muon_step(s["weight"], s["grad"], s["momentum"], lr=LR, momentum_decay=MU, weight_decay=WD, nesterov=True, steps=s["steps"], eps=EPS)
    return {"weight": s["weight"], "momentum": s["momentum"]}


@torch.no_grad()
def run(state):
    if own:
        return _own(state)
    op = state["op"]
    if op in ("conv_train", "conv_prompt"):
        return _plain_conv(state)
    if op in ("scan_prompt", "scan_train"):
        return _plain_scan(state)
    return _plain_step(state) if op == "step" else _plain_muon(state)


# ------------------------------------------------------------------------------------------- work
def work(case):
    op, e = case["op"], 4 if case["type"] == "f32" else 2
    if op in ("ortho", "muon"):
        k, m, n = case["count"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # the Gram matrix and its square are symmetric: half of each has to be computed
        flops = k * case["steps"] * (m * (m + 1) * n + m * (m + 1) * m + 2 * m * m * n)
        return {"bytes": k * m * n * (2 * e if op == "ortho" else 3 * e + 8), "flops": flops}
    b, c, length = case["batch"], case["channels"], case.get("length", 1)
    x, w, n = b * length * c, case.get("width", 0), case.get("states", 0)
    window = b * (w - 1) * c * e if w else 0
    if op == "conv_prompt":
        return {"bytes": 2 * x * e + 2 * window + 4 * c * (w + 1), "flops": x * (2 * w + 4)}
    if op == "conv_train":
        return {"bytes": 4 * x * e + 2 * window + 8 * c * (w + 1), "flops": x * (6 * w + 14)}
    rows, state, fixed = 2 * b * length * n * e, 4 * b * c * n, 4 * c * (n + 2)
    if op == "scan_prompt":
        return {"bytes": 4 * x * e + rows + 2 * state + fixed, "flops": 7 * x * n}
    if op == "scan_train":
        return {"bytes": 8 * x * e + 2 * rows + 3 * state + 2 * fixed, "flops": 23 * x * n}
    return {"bytes": 5 * x * e + rows + 2 * state + fixed + 2 * window + 4 * c * (w + 1), "flops": 7 * x * n + x * (2 * w + 4)}


# ------------------------------------------------------------------------------- 64-bit definition
def _exact_conv(s, train):
    d = torch.float64
    x, win, wt, bias = s["x"].to(d), s["window"].to(d), s["weight"].to(d), s["bias"].to(d)
    w, length = wt.shape[1], x.shape[1]
    full = torch.cat((win, x), 1)
    pre = bias.expand_as(x).clone()
    for j in range(w):
        pre += full[:, j:j + length] * wt[:, j]
    gate = torch.sigmoid(pre)
    if not train:
        return {"y": pre * gate, "window": full[:, length:]}
    g = s["gy"].to(d) * (gate + pre * gate * (1 - gate))
    gfull = torch.zeros_like(full)
    gw = torch.zeros_like(wt)
    for j in range(w):
        gfull[:, j:j + length] += g * wt[:, j]
        gw[:, j] = (full[:, j:j + length] * g).sum((0, 1))
    return {"y": pre * gate, "gx": gfull[:, w - 1:], "gwindow": gfull[:, :w - 1], "gweight": gw, "gbias": g.sum((0, 1))}


def _exact_scan(s, train):
    d = torch.float64
    u, z, bt, ct = (s[k].to(d) for k in ("u", "z", "B", "C"))
    A, D, h = s["A"].to(d), s["D"].to(d), s["state"].to(d)
    raw = s["delta"].to(d) + s["delta_bias"].to(d)
    step = torch.nn.functional.softplus(raw, threshold=60)
    length = u.shape[1]
    y, seen = torch.empty_like(u), []
    for t in range(length):
        if train:
            seen.append(h)
        h = torch.exp(step[:, t, :, None] * A) * h + (step[:, t] * u[:, t])[..., None] * bt[:, t, None, :]
        y[:, t] = torch.einsum("bcn,bn->bc", h, ct[:, t]) + D * u[:, t]
    sig = torch.sigmoid(z)
    if not train:
        return {"out": y * z * sig, "state": h}
    go = s["gout"].to(d)
    gy, gz = go * z * sig, go * y * (sig + z * sig * (1 - sig))
    gu, gstep, gb, gc, gA = torch.empty_like(u), torch.empty_like(u), torch.empty_like(bt), torch.empty_like(ct), torch.zeros_like(A)
    adj, last = torch.zeros_like(h), h
    for t in reversed(range(length)):
        gc[:, t] = torch.einsum("bcn,bc->bn", h, gy[:, t])
        h = seen.pop()
        adj = adj + gy[:, t, :, None] * ct[:, t, None, :]
        keep = torch.exp(step[:, t, :, None] * A)
        through = torch.einsum("bcn,bn->bc", adj, bt[:, t])
        gb[:, t] = torch.einsum("bcn,bc->bn", adj, step[:, t] * u[:, t])
        gu[:, t] = step[:, t] * through + D * gy[:, t]
        p = adj * keep * h
        gstep[:, t] = (p * A).sum(-1) + u[:, t] * through
        gA += (p * step[:, t, :, None]).sum(0)
        adj = adj * keep
    graw = gstep * torch.sigmoid(raw)
    return {"out": y * z * sig, "state": last, "gu": gu, "gdelta": graw, "gz": gz, "gB": gb, "gC": gc, "gA": gA,
            "gD": (gy * u).sum((0, 1)), "gdelta_bias": graw.sum((0, 1)), "gstate": adj}


def _exact_step(s):
    d, dt = torch.float64, s["dtype"]
    full = torch.cat((s["window"], s["x"][:, None]), 1)
    pre = torch.einsum("bwc,cw->bc", full.to(d), s["weight"].to(d)) + s["bias"].to(d)
    u = pre * torch.sigmoid(pre)
    v = u.to(dt).to(d)                                            # the scan reads what the convolution stored
    step = torch.nn.functional.softplus(s["delta"].to(d) + s["delta_bias"].to(d), threshold=60)
    h = torch.exp(step[..., None] * s["A"].to(d)) * s["state"].to(d) + (step * v)[..., None] * s["B"].to(d)[:, None]
    z = s["z"].to(d)
    out = (torch.einsum("bcn,bn->bc", h, s["C"].to(d)) + s["D"].to(d) * v) * z * torch.sigmoid(z)
    return {"u": u, "out": out, "window": full[:, 1:].to(d), "state": h}


def _exact_muon(s):
    d = torch.float64
    g = s["grad"].to(d)
    if s["op"] == "muon":
        mom = s["momentum"].to(d) * MU + g
        g = g + MU * mom
    x = g / (torch.linalg.vector_norm(g, dim=(1, 2), keepdim=True) + EPS)
    wide = x.shape[2] > x.shape[1]
    for _ in range(s["steps"]):
        if wide:
            gram = x @ x.mT
            x = NS_A * x + (NS_B * gram + NS_C * gram @ gram) @ x
        else:
            gram = x.mT @ x
            x = NS_A * x + x @ (NS_B * gram + NS_C * gram @ gram)
    if s["op"] == "ortho":
        return {"out": x}
    rate = LR * max(1.0, x.shape[1] / x.shape[2]) ** 0.5
    return {"weight": s["weight"].to(d) * (1 - LR * WD) - rate * x, "momentum": mom}


@torch.no_grad()
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("conv_train", "conv_prompt"):
        return _exact_conv(s, op == "conv_train")
    if op in ("scan_prompt", "scan_train"):
        return _exact_scan(s, op == "scan_train")
    return _exact_step(s) if op == "step" else _exact_muon(s)
