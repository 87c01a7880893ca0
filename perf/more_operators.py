"""The retention mixer of a space-time network, as cases to be measured.

A network that marches a field along an axis of the grid can mix each row of nodes with linear attention
that forgets: queries and keys are normalised and rotated by their position, head by head, and a matrix
state for each head, which decays from node to node, carries what was seen.  Each case is one call, or one
forward and backward pair of calls, of those operators:

    rotary       rotation of queries and keys by their position, forward (and gradients, "train")
    norm_rotary  norm of each head's query and key and the rotation in one pass, forward (and gradients)
    linear       linear attention with a decay for each head, forward with the state left for the next
                 node (and gradients)
    linear_step  one node for each row: the state moved on by one

`own = False` computes the plain form in 32 bits with elementary torch operations, `own = True` calls
this package.  `exact` restates each operator in 64 bits, the attention one node after the other.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
BASE = 10000.0
CHUNK = 64                                     # nodes that the plain form takes at once


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # inference on a 256 x 128 space-time grid, one row of 128 time nodes for each x: latency
        {"name": "rotary_f32_grid", "op": "rotary", "train": False, "type": "f32", "batch": 256, "length": 128, "heads": 4, "k_heads": 4, "dim": 32,
         "rotary": 32, "interleaved": False, "offset": 0, "stretch": 1.0, "positions": False},
        # training far along long rows: half of each head turns, neighbours in pairs, positions stretched, fewer keys than queries
        {"name": "rotary_train_bf16_far", "op": "rotary", "train": True, "type": "bf16", "batch": 4, "length": 4096, "heads": 16, "k_heads": 4,
         "dim": 128, "rotary": 64, "interleaved": True, "offset": 1000000, "stretch": 8.0, "positions": False},
        # a small network's training step: odd rows, a head width that is no multiple of 8
        {"name": "norm_rotary_train_f32_odd", "op": "norm_rotary", "train": True, "type": "f32", "batch": 5, "length": 1001, "heads": 3, "k_heads": 3,
         "dim": 44, "rotary": 22, "interleaved": False, "offset": 0, "stretch": 1.0, "positions": True},
        # training of a wide network on long rows: as much as memory can move
        {"name": "norm_rotary_train_bf16_wide", "op": "norm_rotary", "train": True, "type": "bf16", "batch": 8, "length": 4096, "heads": 16,
         "k_heads": 16, "dim": 128, "rotary": 128, "interleaved": False, "offset": 0, "stretch": 1.0, "positions": False},
        # marching all rows of a 256-node axis by one node, each at a position of its own: latency
        {"name": "norm_rotary_bf16_rows", "op": "norm_rotary", "train": False, "type": "bf16", "batch": 256, "length": 1, "heads": 32, "k_heads": 8,
         "dim": 128, "rotary": 128, "interleaved": False, "offset": 0, "stretch": 1.0, "positions": True},
        # inference of a small network on one row of 100 time nodes: latency
        {"name": "linear_f32_short", "op": "linear", "train": False, "type": "f32", "batch": 1, "length": 100, "heads": 4, "dk": 32, "dv": 32},
        # one long row: few heads for the whole GPU, so the axis has to be split
        {"name": "linear_bf16_long", "op": "linear", "train": False, "type": "bf16", "batch": 1, "length": 16384, "heads": 16, "dk": 64, "dv": 64},
        # many rows of a wide network: the throughput case
        {"name": "linear_bf16_wide", "op": "linear", "train": False, "type": "bf16", "batch": 8, "length": 2048, "heads": 32, "dk": 128, "dv": 128},
        # a training step on the 256 x 128 grid
        {"name": "linear_train_f32_grid", "op": "linear", "train": True, "type": "f32", "batch": 256, "length": 128, "heads": 4, "dk": 32, "dv": 32},
        # a training step of a wide network on long rows
        {"name": "linear_train_bf16_wide", "op": "linear", "train": True, "type": "bf16", "batch": 4, "length": 4096, "heads": 16, "dk": 128, "dv": 128},
        # marching one row by one node: latency
        {"name": "linear_step_f32_one", "op": "linear_step", "type": "f32", "batch": 1, "heads": 8, "dk": 64, "dv": 64},
        # marching all rows of a 256-node axis by one node: the states' traffic
        {"name": "linear_step_bf16_rows", "op": "linear_step", "type": "bf16", "batch": 256, "heads": 32, "dk": 128, "dv": 128},
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng):
    """The width of a head: a usual one as often as any."""
    return rng.choice((32, 64, 64, 128)) if rng.random() < 0.6 else _between(rng, 8, 128)


def draw(rng):
    op = rng.choice(("rotary", "norm_rotary", "linear", "linear", "linear_step"))
    case = {"op": op, "type": rng.choice(("f32", "bf16"))}
    if op in ("rotary", "norm_rotary"):
        case["train"] = rng.random() < 0.5
        dim = _width(rng)
        k_heads = rng.choice((1, 2, 3, 4, 8, 16))
        heads = k_heads * rng.choice((1, 1, 2, 4))
        length = _between(rng, 1, 16384)
        room = (1 << (25 if case["train"] else 26)) // (dim * (heads + k_heads))
        length = min(length, room)
        case |= {"batch": _between(rng, 1, max(1, min(256, room // length))), "length": length, "heads": heads, "k_heads": k_heads, "dim": dim,
                 "rotary": 2 * max(1, int(dim * rng.choice((0.25, 0.5, 1.0, 1.0)) / 2)), "interleaved": rng.random() < 0.5,
                 "offset": rng.choice((0, 0, 777, 1000000)), "stretch": rng.choice((1.0, 1.0, 4.0)), "positions": rng.random() < 0.5}
    elif op == "linear":
        case["train"] = rng.random() < 0.5
        dk, dv, heads = _width(rng), _width(rng), rng.choice((1, 3, 4, 8, 16, 32))
        room = (1 << (25 if case["train"] else 26)) // (max(dk, dv) * heads)
        length = _between(rng, 1, min(16384, room))
        # a row's state is as much as some 64 to 128 nodes of it
        case |= {"batch": _between(rng, 1, max(1, min(256, room // (length + 128)))), "length": length, "heads": heads, "dk": dk, "dv": dv}
    else:
        case |= {"batch": _between(rng, 1, 256), "heads": rng.choice((1, 3, 4, 8, 16, 32)), "dk": _width(rng), "dv": _width(rng)}
    return case


# ----------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    dt, op, b = TYPES[case["type"]], case["op"], case["batch"]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE) * scale

    s = {"op": op, "dtype": dt, "train": case.get("train", False)}
    if op in ("rotary", "norm_rotary"):
        length, hq, hk, dim = case["length"], case["heads"], case["k_heads"], case["dim"]
        both = normal(b, length, hq + hk, dim).to(dt)             # the projection that gives queries and keys
        pairs = torch.arange(case["rotary"] // 2, device=DEVICE, dtype=torch.float64)
        s |= {"q": both[:, :, :hq], "k": both[:, :, hq:], "interleaved": case["interleaved"], "offset": case["offset"],
              "inv_freq": (BASE ** (-2 * pairs / case["rotary"]) / case["stretch"]).to(torch.float32)}
        s["positions"] = None
        if case["positions"]:                                     # rows that start each at a node of its own
            start = torch.randint(0, 4096, (b, 1), generator=g, device=DEVICE)
            s["positions"] = start + torch.arange(length, device=DEVICE)
        if op == "norm_rotary":
            s |= {"q_weight": 1 + normal(dim, scale=0.1), "k_weight": 1 + normal(dim, scale=0.1)}
        if s["train"]:
            s |= {"gq": normal(b, length, hq, dim).to(dt), "gk": normal(b, length, hk, dim).to(dt)}
        return s
    h, dk, dv = case["heads"], case["dk"], case["dv"]
    # a retention layer's decays: heads that see from some 32 to some 512 nodes back
    far = torch.linspace(math.log(32.0), math.log(512.0), h, device=DEVICE, dtype=torch.float64)
    s |= {"log_decay": torch.log1p(-torch.exp(-far)).to(torch.float32), "scale": dk ** -0.5, "state": normal(b, h, dk, dv, scale=2.0)}
    lead = (b,) if op == "linear_step" else (b, case["length"])
    both = normal(*lead, 2 * h, dk).to(dt)
    s |= {"q": both[..., :h, :], "k": both[..., h:, :], "v": normal(*lead, h, dv).to(dt)}
    if s["train"]:
        s |= {"go": normal(*lead, h, dv).to(dt), "gstate": normal(b, h, dk, dv, scale=0.1)}
    return s


# ------------------------------------------------------------------------------------ plain forms
def _cos_sin(s, length):
    """Of the angle position * frequency, formed in 64 bits: (batch or 1, length, 1, pairs)."""
    at = torch.arange(length, device=DEVICE).unsqueeze(0) if s["positions"] is None else s["positions"]
    angle = (at + s["offset"]).to(torch.float64).unsqueeze(-1) * s["inv_freq"].to(torch.float64)
    return torch.cos(angle).to(torch.float32).unsqueeze(2), torch.sin(angle).to(torch.float32).unsqueeze(2)


def _turn(x, cos, sin, interleaved):
    n = cos.shape[-1]
    a, b, rest = (x[..., 0:2 * n:2], x[..., 1:2 * n:2], x[..., 2 * n:]) if interleaved else (x[..., :n], x[..., n:2 * n], x[..., 2 * n:])
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((c, d), -1).flatten(-2) if interleaved else torch.cat((c, d), -1)
    return torch.cat((turned, rest), -1)


def _plain_rotary(s):
    f, dt, turn = torch.float32, s["dtype"], s["interleaved"]
    cos, sin = _cos_sin(s, s["q"].shape[1])
    out = {"q": _turn(s["q"].to(f), cos, sin, turn).to(dt), "k": _turn(s["k"].to(f), cos, sin, turn).to(dt)}
    if s["train"]:
        out |= {"gq": _turn(s["gq"].to(f), cos, -sin, turn).to(dt), "gk": _turn(s["gk"].to(f), cos, -sin, turn).to(dt)}
    return out


def _norm_turn(x, w, cos, sin, turn):
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return _turn(x * r * w, cos, sin, turn)


def _norm_turn_back(g, x, w, cos, sin, turn):
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    g, unit = _turn(g, cos, -sin, turn), x * r
    gw = g * w
    return r * (gw - unit * (gw * unit).mean(-1, keepdim=True)), (g * unit).sum((0, 1, 2))


def _plain_norm_rotary(s):
    f, dt, turn = torch.float32, s["dtype"], s["interleaved"]
    cos, sin = _cos_sin(s, s["q"].shape[1])
    q, k = s["q"].to(f), s["k"].to(f)
    out = {"q": _norm_turn(q, s["q_weight"], cos, sin, turn).to(dt), "k": _norm_turn(k, s["k_weight"], cos, sin, turn).to(dt)}
    if s["train"]:
        gq, gqw = _norm_turn_back(s["gq"].to(f), q, s["q_weight"], cos, sin, turn)
        gk, gkw = _norm_turn_back(s["gk"].to(f), k, s["k_weight"], cos, sin, turn)
        out |= {"gq": gq.to(dt), "gk": gk.to(dt), "gq_weight": gqw, "gk_weight": gkw}
    return out


def _powers(log_decay, n):
    """decay^n for each head, formed in 64 bits: (heads, *n.shape); 0 where n is negative."""
    d = log_decay.to(torch.float64).view(-1, *[1] * n.dim())
    return torch.where(n < 0, 0.0, torch.exp(d * n.clamp(min=0))).to(torch.float32)


def _attend(q, k, v, log_decay, start, shift):
    """sum over j <= i of decay^(i-j) (q_i . k_j) v_j + decay^(i+1-shift) q_i start, and the sum over j of
    decay^(length-1-j+shift) k_j v_j^T; tensors (batch, heads, length, dim)."""
    b, h, length, dk = q.shape
    n = -(-length // CHUNK)
    pad = n * CHUNK - length                                       # empty nodes ahead of the row
    cut = [torch.cat((t.new_zeros(b, h, pad, t.shape[-1]), t), 2).view(b, h, n, CHUNK, t.shape[-1]) for t in (q, k, v)]
    at = torch.arange(CHUNK, device=DEVICE)
    near = (cut[0] @ cut[1].transpose(-1, -2)) * _powers(log_decay, at[:, None] - at).unsqueeze(1) @ cut[2]
    local = (cut[1] * _powers(log_decay, CHUNK - 1 - at + shift)[:, None, :, None]).transpose(-1, -2) @ cut[2]     # of each chunk
    ends = torch.arange(n + 1, device=DEVICE)
    carry = _powers(log_decay, (ends[:, None] - 1 - ends[:n]) * CHUNK)                                             # (heads, n + 1, n)
    states = (carry @ local.flatten(3)).view(b, h, n + 1, dk, -1)
    far = (cut[0] * _powers(log_decay, at + 1 - shift)[:, None, :, None]) @ states[:, :, :n]
    out = (near + far).view(b, h, n * CHUNK, -1)[:, :, pad:]
    every = torch.arange(length, device=DEVICE)
    return out + (q * _powers(log_decay, every + 1 - shift)[:, :, None]) @ start, states[:, :, n]


def _plain_linear(s):
    f, dt, d, scale = torch.float32, s["dtype"], s["log_decay"], s["scale"]
    q, k, v = (s[n].to(f).transpose(1, 2) for n in "qkv")
    q, back = q * scale, lambda t: t.transpose(1, 2).to(dt)        # noqa: E731
    whole = _powers(d, torch.tensor([q.shape[2]], device=DEVICE)).unsqueeze(-1)
    o, last = _attend(q, k, v, d, s["state"], 0)
    out = {"o": back(o), "state": last + whole * s["state"]}
    if s["train"]:
        go = s["go"].to(f).transpose(1, 2)
        gq, _ = _attend(go, v, k, d, s["state"].transpose(-1, -2), 0)
        q, k, v, go = (t.flip(2) for t in (q, k, v, go))
        gk, _ = _attend(v, go, q, d, s["gstate"].transpose(-1, -2), 1)
        gv, first = _attend(k, q, go, d, s["gstate"], 1)
        out |= {"gq": back(gq * scale), "gk": back(gk.flip(2)), "gv": back(gv.flip(2)), "gstate": first + whole * s["gstate"]}
    return out


def _plain_step(s):
    f = torch.float32
    q, k, v = (s[n].to(f) for n in "qkv")
    decay = torch.exp(s["log_decay"].to(torch.float64)).to(f)[:, None, None]
    s["state"].copy_(decay * s["state"] + k.unsqueeze(-1) * v.unsqueeze(-2))
    o = (s["scale"] * q).unsqueeze(-2) @ s["state"]
    return {"o": o.squeeze(-2).to(s["dtype"]), "state": s["state"]}


# --------------------------------------------------------------------------------- the package's
def _own(s):
    from paper_2607_18020_b200 import sequence
    op = s["op"]
    if op == "rotary":
        how = {"positions": s["positions"], "offset": s["offset"], "interleaved": s["interleaved"]}
        q, k = sequence.rotary_fwd(s["q"], s["k"], s["inv_freq"], **how)
        if not s["train"]:
            return {"q": q, "k": k}
        gq, gk = sequence.rotary_bwd(s["gq"], s["gk"], s["inv_freq"], **how)
        return {"q": q, "k": k, "gq": gq, "gk": gk}
    if op == "norm_rotary":
        args = (s["q"], s["k"], s["q_weight"], s["k_weight"], s["inv_freq"])
        how = {"positions": s["positions"], "offset": s["offset"], "interleaved": s["interleaved"], "eps": EPS}
        q, k = sequence.norm_rotary_fwd(*args, **how)
        if not s["train"]:
            return {"q": q, "k": k}
        g = sequence.norm_rotary_bwd(s["gq"], s["gk"], *args, **how)
        return {"q": q, "k": k, "gq": g.q, "gk": g.k, "gq_weight": g.q_weight, "gk_weight": g.k_weight}
    if op == "linear":
        args = (s["q"], s["k"], s["v"], s["log_decay"])
        o, last = sequence.linear_attention_fwd(*args, scale=s["scale"], state=s["state"])
        if not s["train"]:
            return {"o": o, "state": last}
        g = sequence.linear_attention_bwd(s["go"], *args, scale=s["scale"], state=s["state"], gstate=s["gstate"])
        return {"o": o, "state": last, "gq": g.q, "gk": g.k, "gv": g.v, "gstate": g.state}
    o = sequence.linear_attention_step(s["state"], s["q"], s["k"], s["v"], s["log_decay"], scale=s["scale"])
    return {"o": o, "state": s["state"]}


@torch.no_grad()
def run(state):
    if own:
        return _own(state)
    return {"rotary": _plain_rotary, "norm_rotary": _plain_norm_rotary, "linear": _plain_linear, "linear_step": _plain_step}[state["op"]](state)


# ------------------------------------------------------------------------------------------- work
def work(case):
    op, e, b = case["op"], 4 if case["type"] == "f32" else 2, case["batch"]
    if op in ("rotary", "norm_rotary"):
        tokens = b * case["length"]
        x = tokens * (case["heads"] + case["k_heads"]) * case["dim"]
        at = 8 * tokens if case["positions"] else 0
        if op == "rotary":
            return {"bytes": (4 if case["train"] else 2) * x * e + at, "flops": (6 if case["train"] else 3) * x}
        # the gradients take the inputs and the upstream gradients in and give as much as the inputs
        return {"bytes": (4 if case["train"] else 2) * x * e + at + (16 if case["train"] else 8) * case["dim"], "flops": (18 if case["train"] else 6) * x}
    h, dk, dv = case["heads"], case["dk"], case["dv"]
    nodes, state = b * h * case.get("length", 1), 4 * b * h * dk * dv
    qkvo = 2 * nodes * (dk + dv) * e
    # node by node: the state is moved on (3 operations an element) and read (2); each gradient does as much
    if case.get("train"):
        # in: q, k, v, go and both states; out: o, gq, gk, gv and both states
        return {"bytes": 4 * nodes * (dk + dv) * e + 4 * state + 4 * h, "flops": 17 * nodes * dk * dv}
    return {"bytes": qkvo + 2 * state + 4 * h, "flops": 5 * nodes * dk * dv}


# ------------------------------------------------------------------------------- 64-bit definition
def _exact_turn(x, s, sign):
    """Each pair as a complex number times e^(i angle)."""
    n = s["inv_freq"].shape[0]
    at = s["positions"] if s["positions"] is not None else torch.arange(x.shape[1], device=DEVICE)[None]
    angle = sign * (at + s["offset"]).double()[:, :, None, None] * s["inv_freq"].double()
    y = x.clone()
    i = torch.arange(n, device=DEVICE)
    first, second = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + n)
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_rotary(s):
    out = {"q": _exact_turn(s["q"].double(), s, 1), "k": _exact_turn(s["k"].double(), s, 1)}
    if s["train"]:
        out |= {"gq": _exact_turn(s["gq"].double(), s, -1), "gk": _exact_turn(s["gk"].double(), s, -1)}
    return out


def _exact_norm_rotary(s):
    out = {}
    for n in "qk":
        x, w = s[n].double(), s[n + "_weight"].double()
        size = ((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
        out[n] = _exact_turn(x / size * w, s, 1)
        if s["train"]:
            g = _exact_turn(s["g" + n].double(), s, -1)
            out["g%s_weight" % n] = (g * x / size).sum((0, 1, 2))
            along = (g * w * x).sum(-1, keepdim=True) / x.shape[-1]
            out["g" + n] = g * w / size - x * along / size ** 3
    return out


def _exact_linear(s):
    decay = torch.exp(s["log_decay"].double())[:, None, None]
    q, k, v = (s[n].double() for n in "qkv")
    scale, length = s["scale"], q.shape[1]
    S, o, gq = s["state"].double(), torch.empty_like(v), torch.empty_like(q)
    go = s["go"].double() if s["train"] else None
    for t in range(length):
        S = S * decay + k[:, t, :, :, None] * v[:, t, :, None, :]
        o[:, t] = scale * (q[:, t, :, None, :] @ S)[:, :, 0]
        if s["train"]:
            gq[:, t] = scale * (S @ go[:, t, :, :, None])[..., 0]
    out = {"o": o, "state": S}
    if s["train"]:
        G, gk, gv = s["gstate"].double(), torch.empty_like(k), torch.empty_like(v)
        for t in range(length - 1, -1, -1):
            G = G + scale * q[:, t, :, :, None] * go[:, t, :, None, :]
            gk[:, t] = (G @ v[:, t, :, :, None])[..., 0]
            gv[:, t] = (k[:, t, :, None, :] @ G)[:, :, 0]
            G = G * decay
        out |= {"gq": gq, "gk": gk, "gv": gv, "gstate": G}
    return out


def _exact_step(s):
    S = torch.exp(s["log_decay"].double())[:, None, None] * s["state"].double() + torch.einsum("bhi,bhj->bhij", s["k"].double(), s["v"].double())
    return {"o": torch.einsum("bhi,bhij->bhj", s["q"].double() * s["scale"], S), "state": S}


@torch.no_grad()
def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "norm_rotary": _exact_norm_rotary, "linear": _exact_linear, "linear_step": _exact_step}[case["op"]](s)
