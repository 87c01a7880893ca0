"""Causal convolution and selective scan against the 64-bit forms: types, odd sizes, strides, short and
long rows, states handed on, single nodes, gradients, and what happens with infinities and NaN."""
import pytest

torch = pytest.importorskip("torch")
from seq_util import GuardedTorch, check, conv_ref, d64, rel, scan_ref

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


@pytest.fixture
def guard(monkeypatch):
    from paper_2607_18020_b200 import sequence
    g = GuardedTorch()
    monkeypatch.setattr(sequence, "torch", g)
    yield g
    torch.cuda.synchronize()
    g.check()


# ------------------------------------------------------------------------------------- convolution
CONV = [  # batch, length, channels, width, strided view, state, bias, silu
    (1, 1, 1, 4, False, True, True, True), (2, 3, 5, 4, False, True, True, True), (1, 2, 128, 3, True, True, True, False),
    (3, 17, 33, 2, True, False, True, True), (2, 130, 64, 4, True, True, False, True), (2, 128, 256, 4, False, False, False, True),
    (1, 300, 132, 1, True, True, True, True), (5, 259, 40, 3, False, True, True, True), (2, 0, 12, 4, False, True, True, True),
    (0, 9, 12, 4, False, True, True, True), (1, 1025, 20, 4, True, True, True, True),
]


def conv_inputs(case, dtype, seed=3):
    batch, length, channels, width, view, state, bias, silu = case
    r = gen(seed)
    x = r(batch, length, 2 * channels).to(dtype)[..., channels:] if view else r(batch, length, channels).to(dtype)
    w, b = 0.5 * r(channels, width), 0.5 * r(channels) if bias else None
    s = r(batch, width - 1, channels).to(dtype) if state else None
    return x, w, b, s, silu, r(batch, length, channels).to(dtype), r(batch, width - 1, channels).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CONV)
def test_conv_forward_and_gradients(case, dtype, guard):
    from paper_2607_18020_b200 import sequence as Q
    x, w, b, s, silu, gy, gs = conv_inputs(case, dtype)
    y, left = Q.causal_conv_fwd(x, w, b, s, silu)
    g = Q.causal_conv_bwd(gy, x, w, b, s, silu, gs)
    leaves = [t.requires_grad_(True) if t is not None else None for t in map(d64, (x, w, b, s))]
    ry, rleft = conv_ref(*leaves, silu)
    check("y", y, ry)
    assert torch.equal(left.double().cpu(), rleft.detach())        # copied, not computed
    want = torch.autograd.grad([ry, rleft], [t for t in leaves if t is not None], [d64(gy), d64(gs)])
    got = [t for t in (g.x, g.weight, g.bias, g.state) if t is not None]
    assert len(got) == len(want)
    for name, a, e in zip("xwbs", got, want):
        check("g" + name, a, e)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("channels,width", [(1, 4), (37, 3), (256, 4), (64, 1), (130, 2)])
def test_conv_steps_continue_a_row(dtype, channels, width, guard):
    from paper_2607_18020_b200 import sequence as Q
    r = gen(5)
    x, w, b = r(3, 9, 2 * channels).to(dtype)[..., :channels], 0.5 * r(channels, width), r(channels)
    y, left = Q.causal_conv_fwd(x, w, b)
    window = torch.zeros(3, width - 1, channels, dtype=dtype, device="cuda")
    ys = [Q.causal_conv_step(x[:, t], window, w, b) for t in range(9)]
    assert rel(torch.stack(ys, 1), y) <= 1e-6 or dtype != torch.float32
    check("steps", torch.stack(ys, 1), conv_ref(d64(x), d64(w), d64(b), None, True)[0])
    assert torch.equal(window, left)


def test_conv_pieces_of_a_row_agree_with_the_row():
    from paper_2607_18020_b200 import sequence as Q
    r = gen(6)
    x, w, b = r(2, 203, 48), 0.5 * r(48, 4), r(48)
    y, left = Q.causal_conv_fwd(x, w, b)
    at, state, ys = 0, None, []
    for n in (1, 2, 60, 0, 140):
        p, state = Q.causal_conv_fwd(x[:, at:at + n], w, b, state)
        ys.append(p)
        at += n
    assert torch.equal(torch.cat(ys, 1), y) and torch.equal(state, left)


def test_conv_nan_and_infinity_stay_within_reach():
    from paper_2607_18020_b200 import sequence as Q
    r = gen(7)
    x, w = r(1, 64, 32), 0.5 * r(32, 4)
    clean, _ = Q.causal_conv_fwd(x, w)
    x[0, 20, 3], x[0, 40, 7] = float("nan"), float("inf")
    y, _ = Q.causal_conv_fwd(x, w)
    same = torch.ones_like(y, dtype=torch.bool)
    same[0, 20:24, 3] = False
    same[0, 40:44, 7] = False
    assert torch.equal(y[same], clean[same])
    assert bool(torch.isnan(y[0, 20:24, 3]).all())


def test_conv_autograd_differences():
    """Directional differences of the fp32 kernels; the step balances rounding (1e-7/h) and curvature (h^2)."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(8)
    t = [r(2, 21, 12), 0.5 * r(12, 4), r(12), r(2, 3, 12)]
    wts = r(2, 21, 12).double()
    f = lambda *a: (Q.causal_conv(*a).double() * wts).sum()    # noqa: E731
    leaves = [v.clone().requires_grad_(True) for v in t]
    grads = torch.autograd.grad(f(*leaves), leaves)
    h = 1e-2
    for k, g in enumerate(grads):
        d = r(*t[k].shape)
        hi, lo = ([v + s * h * d if i == k else v for i, v in enumerate(t)] for s in (1, -1))
        diff = float(f(*hi) - f(*lo)) / (2 * h)
        along = float((g.double() * d.double()).sum())
        scale = float(torch.linalg.vector_norm(g.double()) * torch.linalg.vector_norm(d.double()))
        assert abs(diff - along) <= 1e-3 * scale, (k, diff, along)


# -------------------------------------------------------------------------------------------- scan
SCAN = [  # batch, length, channels, states, strided views, state, extras (D, z, bias), softplus
    (1, 1, 1, 1, False, True, True, True), (2, 5, 3, 4, False, True, True, True), (1, 16, 64, 16, True, True, True, True),
    (2, 33, 70, 16, True, True, True, True), (1, 100, 32, 5, True, False, False, False), (2, 64, 130, 8, False, True, True, True),
    (1, 47, 40, 24, True, True, True, True), (1, 70, 9, 64, True, True, True, True), (2, 31, 17, 33, False, False, True, True),
    (2, 0, 6, 16, False, True, True, True), (0, 7, 6, 16, False, True, True, True), (1, 517, 36, 16, True, True, True, True),
    (3, 257, 20, 12, True, True, False, True),
]


def scan_inputs(case, dtype, seed=11):
    batch, length, channels, n, view, state, extras, softplus = case
    r = gen(seed)

    def act(c):
        return r(batch, length, 2 * c + 3).to(dtype)[..., 3:c + 3] if view else r(batch, length, c).to(dtype)
    u, delta, B, C = act(channels), act(channels), act(n), act(n)
    if not softplus:
        delta = (0.1 * torch.rand(batch, length, channels, device="cuda")).to(dtype)
    A = -(0.5 + torch.rand(channels, n, device="cuda") * n)
    D, z, bias = (r(channels), act(channels), r(channels) - 2) if extras else (None, None, None)
    s = r(batch, channels, n) if state else None
    return (u, delta, A, B, C, D, z, bias), softplus, s, r(batch, length, channels).to(dtype), r(batch, channels, n)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", SCAN)
def test_scan_forward_and_gradients(case, dtype, guard):
    from paper_2607_18020_b200 import sequence as Q
    t, softplus, s, go, gl = scan_inputs(case, dtype)
    out, last, kept = Q.selective_scan_fwd(*t, delta_softplus=softplus, state=s, keep=True)
    g = Q.selective_scan_bwd(go, *t, delta_softplus=softplus, state=s, kept=kept, gstate=gl)
    leaves = [v.requires_grad_(True) if v is not None else None for v in map(d64, t)]
    rs = d64(s)
    if rs is not None:
        rs.requires_grad_(True)
    rout, rlast = scan_ref(*leaves, softplus, rs)
    check("out", out, rout)
    check("state", last, rlast)
    names = ["u", "delta", "A", "B", "C", "D", "z", "delta_bias", "state"]
    pairs = [(n, leaf) for n, leaf in zip(names, leaves + [rs]) if leaf is not None]
    want = torch.autograd.grad([rout, rlast], [leaf for _, leaf in pairs], [d64(go), d64(gl)], allow_unused=True)
    for (n, leaf), e in zip(pairs, want):
        check("g" + n, getattr(g, n), torch.zeros_like(leaf) if e is None else e)


@pytest.mark.parametrize("length", [1, 63, 64, 65, 4096, 5003])
def test_scan_long_rows_are_joined(length):
    """One row: cut into chunks.  The pieces have to agree with each other and with the 64-bit form."""
    from paper_2607_18020_b200 import sequence as Q
    t, softplus, s, go, gl = scan_inputs((1, length, 24, 16, False, True, True, True), torch.float32, seed=12)
    t = (t[0], t[1] - 3, -torch.rand(24, 16, device="cuda") * 4) + t[3:]      # decays slow enough to reach across chunks
    out, last, kept = Q.selective_scan_fwd(*t, state=s, keep=True)
    g = Q.selective_scan_bwd(go, *t, state=s, kept=kept, gstate=gl)
    leaves = [v.requires_grad_(True) for v in map(d64, t)]
    rs = d64(s).requires_grad_(True)
    rout, rlast = scan_ref(*leaves, True, rs)
    check("out", out, rout)
    check("state", last, rlast)
    want = torch.autograd.grad([rout, rlast], leaves + [rs], [d64(go), d64(gl)])
    for n, e in zip(["u", "delta", "A", "B", "C", "D", "z", "delta_bias", "state"], want):
        check("g" + n, getattr(g, n), e)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("channels,n", [(1, 1), (37, 16), (256, 16), (20, 40), (64, 64), (50, 7)])
def test_scan_steps_continue_a_row(dtype, channels, n, guard):
    from paper_2607_18020_b200 import sequence as Q
    (u, delta, A, B, C, D, z, bias), _, s, _, _ = scan_inputs((3, 7, channels, n, True, True, True, True), dtype, seed=13)
    state = s.clone()
    outs = [Q.selective_scan_step(state, u[:, t], delta[:, t], A, B[:, t], C[:, t], D, z[:, t], bias) for t in range(7)]
    rout, rlast = scan_ref(*map(d64, (u, delta, A, B, C, D, z, bias)), True, d64(s))
    check("out", torch.stack(outs, 1), rout)
    check("state", state, rlast)


def test_scan_broadcast_inputs_and_their_gradients():
    """Rows that share one delta and one B (stride 0): autograd adds the rows' gradients up."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(14)
    u, C = r(3, 20, 16), r(3, 20, 16)
    delta, B = r(1, 20, 16).requires_grad_(True), r(1, 20, 16).requires_grad_(True)
    A = -torch.rand(16, 16, device="cuda") - 0.1
    go = r(3, 20, 16)
    out = Q.selective_scan(u, delta.expand(3, -1, -1), A, B.expand(3, -1, -1), C)
    got = torch.autograd.grad(out, [delta, B], go)
    d2, b2 = d64(delta).requires_grad_(True), d64(B).requires_grad_(True)
    ref, _ = scan_ref(d64(u), d2.expand(3, -1, -1), d64(A), b2.expand(3, -1, -1), d64(C), None, None, None, True, None)
    for a, e in zip(got, torch.autograd.grad(ref, [d2, b2], d64(go))):
        check("shared", a, e)


def test_scan_autograd_differences():
    from paper_2607_18020_b200 import sequence as Q
    (u, delta, A, B, C, D, z, bias), _, s, go, _ = scan_inputs((2, 37, 12, 8, False, True, True, True), torch.float32, seed=15)
    t = [u, delta, A, B, C, D, z, bias, s]
    wts = go.double()
    f = lambda *a: (Q.selective_scan(*a[:8], state=a[8]).double() * wts).sum()    # noqa: E731
    leaves = [v.clone().requires_grad_(True) for v in t]
    grads = torch.autograd.grad(f(*leaves), leaves)
    r, h = gen(16), 3e-3
    for k, g in enumerate(grads):
        d = r(*t[k].shape)
        hi, lo = ([v + sg * h * d if i == k else v for i, v in enumerate(t)] for sg in (1, -1))
        diff = float(f(*hi) - f(*lo)) / (2 * h)
        along = float((g.double() * d.double()).sum())
        scale = float(torch.linalg.vector_norm(g.double()) * torch.linalg.vector_norm(d.double()))
        assert abs(diff - along) <= 1e-3 * scale, (k, diff, along)


def test_scan_nan_stays_in_its_channel_and_behind_its_node():
    from paper_2607_18020_b200 import sequence as Q
    t, _, s, _, _ = scan_inputs((2, 80, 48, 16, False, True, True, True), torch.float32, seed=17)
    clean, last = Q.selective_scan_fwd(*t, state=s)[:2]
    u = t[0].clone()
    u[1, 30, 5] = float("nan")
    out, got = Q.selective_scan_fwd(u, *t[1:], state=s)[:2]
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[1, 30:, 5] = True
    assert torch.equal(out[~hit], clean[~hit]) and bool(torch.isnan(out[hit]).all())
    assert bool(torch.isnan(got[1, 5]).all())
    got[1, 5] = last[1, 5]
    assert torch.equal(got, last)


def test_offsets_past_32_bits():
    """Two rows 2^31 elements apart."""
    from paper_2607_18020_b200 import sequence as Q
    far, channels, length, n = 2 ** 31, 40, 37, 16
    base = torch.empty(far + length * channels, dtype=torch.bfloat16, device="cuda")
    r = gen(21)

    def spread(t):
        v = base.as_strided(t.shape, (far, t.shape[2], 1))
        v.copy_(t)
        return v
    x, w, b = r(2, length, channels).to(torch.bfloat16), 0.5 * r(channels, 4), r(channels)
    gy = r(2, length, channels).to(torch.bfloat16)
    want = Q.causal_conv_fwd(x, w, b)[0]
    gwant = Q.causal_conv_bwd(gy, x, w, b)
    xs = spread(x)
    assert torch.equal(Q.causal_conv_fwd(xs, w, b)[0], want)
    for a, e in zip(Q.causal_conv_bwd(gy, xs, w, b)[:3], gwant[:3]):
        assert torch.equal(a, e)
    t, _, s, go, gl = scan_inputs((2, length, channels, n, False, True, True, True), torch.bfloat16, seed=22)
    out, last, kept = Q.selective_scan_fwd(*t, state=s, keep=True)
    g = Q.selective_scan_bwd(go, *t, state=s, kept=kept, gstate=gl)
    for k in (0, 1, 3, 4, 6):                      # u, delta, B, C, z, one after the other
        far_t = t[:k] + (spread(t[k]),) + t[k + 1:]
        o2, l2, k2 = Q.selective_scan_fwd(*far_t, state=s, keep=True)
        assert torch.equal(o2, out) and torch.equal(l2, last)
        for a, e in zip(Q.selective_scan_bwd(go, *far_t, state=s, kept=k2, gstate=gl), g):
            assert torch.equal(a, e)
    g3 = Q.selective_scan_bwd(spread(go), *t, state=s, kept=kept, gstate=gl)
    assert all(torch.equal(a, e) for a, e in zip(g3, g))
    u1 = spread(t[0])[:, 5]
    s1, s2 = s.clone(), s.clone()
    rest = (t[1][:, 5], t[2], t[3][:, 5], t[4][:, 5])
    assert torch.equal(Q.selective_scan_step(s1, u1, *rest), Q.selective_scan_step(s2, t[0][:, 5], *rest)) and torch.equal(s1, s2)


def test_scan_extreme_steps():
    """delta far below and above: dt underflows to 0 (the state stays) or is large (the state is replaced)."""
    from paper_2607_18020_b200 import sequence as Q
    u, B, C = (torch.ones(1, 3, k, device="cuda") for k in (4, 16, 16))
    A = -torch.ones(4, 16, device="cuda")
    s = torch.full((1, 4, 16), 2.0, device="cuda")
    out, last = Q.selective_scan_fwd(u, torch.full_like(u, -200.0), A, B, C, state=s)[:2]
    assert torch.equal(last, s) and bool((out == 32).all())
    out, last = Q.selective_scan_fwd(u, torch.full_like(u, 300.0), A, B, C, state=s)[:2]
    assert bool((last == 300).all()) and bool((out == 4800).all())


def test_results_do_not_change_from_call_to_call_or_stream_to_stream():
    from paper_2607_18020_b200 import sequence as Q
    t, _, s, go, gl = scan_inputs((2, 700, 100, 16, True, True, True, True), torch.bfloat16, seed=18)

    def once():
        out, last, kept = Q.selective_scan_fwd(*t, state=s, keep=True)
        return (out, last) + tuple(Q.selective_scan_bwd(go, *t, state=s, kept=kept, gstate=gl))
    first = once()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = once()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_calls_can_be_captured_in_a_graph():
    from paper_2607_18020_b200 import sequence as Q
    t, _, s, go, gl = scan_inputs((1, 500, 40, 16, False, True, True, True), torch.float32, seed=19)
    want = Q.selective_scan_fwd(*t, state=s)[0]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = Q.selective_scan_fwd(*t, state=s)[0]
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_refusals():
    from paper_2607_18020_b200 import sequence as Q
    from paper_2607_18020_b200.binding import FpdeError
    t, _, s, go, gl = scan_inputs((2, 5, 6, 16, False, True, True, True), torch.float32)
    u, delta, A, B, C, D, z, bias = t
    with pytest.raises(ValueError):
        Q.selective_scan_fwd(u.cpu(), *t[1:])
    with pytest.raises(ValueError):
        Q.selective_scan_fwd(u.double(), *t[1:])
    with pytest.raises(ValueError):
        Q.selective_scan_fwd(u, delta[:, :4], A, B, C)
    with pytest.raises(ValueError):
        Q.selective_scan_fwd(u, delta.bfloat16(), A, B, C)
    with pytest.raises(ValueError):
        Q.selective_scan_fwd(u, delta, A[:, :8], B, C)
    with pytest.raises(ValueError):
        Q.selective_scan_fwd(u, delta, A, B, C, state=s[:1])
    with pytest.raises(ValueError):
        Q.selective_scan_bwd(go, *t)
    with pytest.raises(FpdeError):
        Q.selective_scan_bwd(go, *t, kept=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(FpdeError):
        n = 65
        Q.selective_scan_fwd(u, delta, -torch.ones(6, n, device="cuda"), torch.ones(2, 5, n, device="cuda"), torch.ones(2, 5, n, device="cuda"))
    with pytest.raises(ValueError):
        Q.selective_scan_step(s.transpose(0, 1).contiguous().transpose(0, 1), u[:, 0], delta[:, 0], A, B[:, 0], C[:, 0])
    x, w = torch.ones(2, 5, 6, device="cuda"), torch.ones(6, 4, device="cuda")
    with pytest.raises(ValueError):
        Q.causal_conv_fwd(x, w[:5])
    with pytest.raises(ValueError):
        Q.causal_conv_fwd(x[0], w)
    with pytest.raises(FpdeError):
        Q.causal_conv_fwd(x, torch.ones(6, 5, device="cuda"))
    with pytest.raises(ValueError):
        Q.causal_conv_step(x[:, 0], torch.ones(2, 2, 6, device="cuda"), w)
