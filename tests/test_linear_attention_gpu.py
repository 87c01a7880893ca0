"""Linear attention with decays against the 64-bit form: types, odd sizes, strides, short and long rows, states handed on,
single nodes, gradients, decays of every size, infinities and NaN, streams and graphs."""
import math

import pytest

torch = pytest.importorskip("torch")
from attention_util import check_attention, linear_ref
from seq_util import GuardedTorch, d64, rel

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
INF = float("inf")


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


def decays(heads):
    """Heads that forget at once, within a few nodes, slowly and never."""
    return torch.tensor([(-0.03, -1.5, 0.0, -INF, -40.0, -1e-4, -0.3)[i % 7] for i in range(heads)], device="cuda")


CASES = [  # batch, length, heads, dk, dv, view, state
    (1, 1, 1, 1, 1, "dense", True), (1, 1, 3, 16, 8, "dense", False), (2, 2, 2, 3, 5, "slice", True), (1, 31, 2, 32, 32, "dense", True),
    (2, 32, 3, 33, 17, "slice", True), (1, 33, 7, 8, 64, "heads first", True), (2, 64, 2, 64, 64, "dense", False), (1, 65, 2, 65, 31, "dense", True),
    (1, 127, 2, 64, 128, "slice", True), (1, 128, 3, 128, 64, "dense", True), (2, 129, 1, 128, 128, "heads first", True),
    (1, 257, 7, 40, 72, "odd", True), (1, 300, 2, 127, 1, "odd", False), (1, 1025, 2, 64, 64, "dense", True), (2, 700, 1, 128, 96, "slice", False),
    (0, 9, 2, 16, 16, "dense", True), (2, 0, 2, 16, 16, "dense", True), (2, 9, 0, 16, 16, "dense", True), (3, 200, 50, 24, 16, "dense", True),
]


def row(r, dtype, batch, length, heads, width, view):
    if view == "slice":
        return r(batch, length, 2 * heads + 1, width + 8).to(dtype)[:, :, 1:heads + 1, 8:]
    if view == "odd":                      # no row starts on more than one element
        return r(batch, length, heads, width + 3).to(dtype)[..., 1:width + 1]
    if view == "heads first":
        return r(batch, heads, length, width).to(dtype).transpose(1, 2)
    return r(batch, length, heads, width).to(dtype)


def inputs(case, dtype, seed=21):
    batch, length, heads, dk, dv, view, state = case
    r = gen(seed)
    q, k, v, go = (row(r, dtype, batch, length, heads, n, view) for n in (dk, dk, dv, dv))
    s = r(batch, heads, dk, dv) if state else None
    return q, k, v, decays(heads), dk ** -0.5, s, go, r(batch, heads, dk, dv)


def wanted(q, k, v, ld, scale, s, go, gs):
    leaves = [None if t is None else t.requires_grad_(True) for t in map(d64, (q, k, v, s))]
    o, last = linear_ref(*leaves[:3], d64(ld), scale, leaves[3])
    grads = torch.autograd.grad([o, last], [t for t in leaves if t is not None], [d64(go), d64(gs)], allow_unused=True)
    return o.detach(), last.detach(), [torch.zeros_like(t) if g is None else g for g, t in zip(grads, leaves)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES)
def test_forward_and_gradients(case, dtype, guard):
    from paper_2607_18020_b200 import sequence as Q
    q, k, v, ld, scale, s, go, gs = inputs(case, dtype)
    o, last = Q.linear_attention_fwd(q, k, v, ld, scale, s)
    g = Q.linear_attention_bwd(go, q, k, v, ld, scale, s, gs)
    ro, rlast, want = wanted(q, k, v, ld, scale, s, go, gs)
    assert o.dtype == dtype and last.dtype == torch.float32
    check_attention("o", o, ro)
    check_attention("state", last, rlast)
    for name, a, e in zip(("gq", "gk", "gv", "gstate"), [t for t in g if t is not None], want):
        check_attention(name, a, e)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,dk,dv", [(1, 1, 1), (3, 16, 24), (2, 33, 5), (5, 64, 64), (2, 128, 128), (1, 7, 127)])
def test_steps_continue_a_row(heads, dk, dv, dtype, guard):
    from paper_2607_18020_b200 import sequence as Q
    r = gen(22)
    q, k, v = (row(r, dtype, 2, 41, heads, n, "slice") for n in (dk, dk, dv))
    ld, scale = decays(heads), 0.3
    o, last = Q.linear_attention_fwd(q[:, :37], k[:, :37], v[:, :37], ld, scale)
    state, steps = last.clone(), []
    for t in range(37, 41):
        steps.append(Q.linear_attention_step(state, q[:, t], k[:, t], v[:, t], ld, scale))
    ro, rlast = linear_ref(d64(q), d64(k), d64(v), d64(ld), scale, None)
    check_attention("steps", torch.stack(steps, 1), ro[:, 37:])
    check_attention("state", state, rlast)


@pytest.mark.parametrize("dtype", TYPES)
def test_pieces_of_a_row_agree_with_the_row(dtype):
    from paper_2607_18020_b200 import sequence as Q
    r = gen(23)
    q, k, v = (r(2, 523, 3, n).to(dtype) for n in (48, 48, 64))
    ld = decays(3)
    state, outs, at = None, [], 0
    for n in (1, 2, 60, 0, 128, 332):
        o, state = Q.linear_attention_fwd(q[:, at:at + n], k[:, at:at + n], v[:, at:at + n], ld, 0.2, state)
        outs.append(o)
        at += n
    ro, rlast = linear_ref(d64(q), d64(k), d64(v), d64(ld), 0.2, None)
    check_attention("o", torch.cat(outs, 1), ro)
    check_attention("state", state, rlast)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_row_is_the_same_alone_and_among_others(dtype):
    """The batch decides how rows are cut, and the results stay within their rounding; the same call gives the same bits."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(24)
    q, k, v = (r(300, 260, 2, 64).to(dtype) for _ in range(3))
    ld = decays(2)
    o, last = Q.linear_attention_fwd(q, k, v, ld, 0.125)
    again, last2 = Q.linear_attention_fwd(q, k, v, ld, 0.125)
    assert torch.equal(o, again) and torch.equal(last, last2)
    alone, end = Q.linear_attention_fwd(q[7:8], k[7:8], v[7:8], ld, 0.125)
    check_attention("alone", alone, o[7:8].double())
    check_attention("state", end, last[7:8].double())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shared_and_broadcast_heads(dtype):
    """Keys and values of one head for all queries, read with a head stride of zero; their gradients are sums over heads."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(25)
    q, k, v, go = r(2, 150, 6, 32).to(dtype), r(2, 150, 1, 32).to(dtype), r(1, 150, 1, 64).to(dtype), r(2, 150, 6, 64).to(dtype)
    ld = decays(6)
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
    o = Q.linear_attention(leaves[0], leaves[1].expand(2, 150, 6, 32), leaves[2].expand(2, 150, 6, 64), ld, 0.2)
    grads = torch.autograd.grad(o, leaves, go)
    ref = [d64(t).requires_grad_(True) for t in (q, k, v)]
    ro, _ = linear_ref(ref[0], ref[1].expand(2, 150, 6, 32), ref[2].expand(2, 150, 6, 64), d64(ld), 0.2, None)
    for name, a, e in zip(("q", "k", "v"), grads, torch.autograd.grad(ro, ref, d64(go))):
        check_attention("g" + name, a, e)


def test_gradients_against_differences():
    """Directional differences of the fp32 forward pass, linear in each input: no curvature, rounding 1e-7 / h."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(26)
    t = [r(2, 45, 2, 24), r(2, 45, 2, 24), r(2, 45, 2, 16), r(2, 2, 24, 16)]
    ld, wo, ws = torch.tensor([-0.05, -0.7], device="cuda"), r(2, 45, 2, 16).double(), r(2, 2, 24, 16).double()

    def f(q, k, v, s):
        o, last = Q.linear_attention(q, k, v, ld, 0.2, s, True)
        return (o.double() * wo).sum() + (last.double() * ws).sum()
    leaves = [x.clone().requires_grad_(True) for x in t]
    for i, g in enumerate(torch.autograd.grad(f(*leaves), leaves)):
        d = r(*t[i].shape)
        hi, lo = ([x + s * d if j == i else x for j, x in enumerate(t)] for s in (1, -1))
        diff, along = float(f(*hi) - f(*lo)) / 2, float((g.double() * d.double()).sum())
        scale = float(torch.linalg.vector_norm(g.double()) * torch.linalg.vector_norm(d.double()))
        assert abs(diff - along) <= 1e-4 * scale, (i, diff, along)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_infinities_and_nan_reach_no_earlier_node(dim, dtype):
    from paper_2607_18020_b200 import sequence as Q
    r = gen(27)
    q, k, v, go = (r(1, 300, 3, dim).to(dtype) for _ in range(4))
    ld = torch.tensor([-0.1, -0.01, 0.0], device="cuda")
    clean, _ = Q.linear_attention_fwd(q, k, v, ld, 0.2)
    cg = Q.linear_attention_bwd(go, q, k, v, ld, 0.2)
    q[0, 50, 0, 3] = float("nan")            # its own node only
    k[0, 141, 1, 5] = INF                    # from there on
    v[0, 200, 2, 7] = -INF                   # from there on, its own feature only
    o, last = Q.linear_attention_fwd(q, k, v, ld, 0.2)
    same = torch.ones_like(o, dtype=torch.bool)
    same[0, 50, 0] = False
    same[0, 141:, 1] = False
    same[0, 200:, 2, 7] = False
    assert torch.equal(o[same], clean[same])
    assert not bool(torch.isfinite(o[~same]).any())
    assert bool(torch.isfinite(last[0, 0]).all()) and bool(torch.isfinite(last[0, 2, :, :7]).all())
    # backwards an upstream value reaches no later node of gk and gv, and no earlier one of gq
    q, k, v = (r(1, 300, 3, dim).to(dtype) for _ in range(3))
    cg = Q.linear_attention_bwd(go, q, k, v, ld, 0.2)
    go[0, 170, 1, 2] = float("nan")
    g = Q.linear_attention_bwd(go, q, k, v, ld, 0.2)
    for a, e in ((g.k, cg.k), (g.v, cg.v)):
        assert torch.equal(a[0, 171:], e[0, 171:]) and torch.equal(a[0, :, [0, 2]], e[0, :, [0, 2]])
    assert torch.equal(g.q[0, :170], cg.q[0, :170]) and torch.equal(g.q[0, 171:], cg.q[0, 171:])
    assert bool(torch.isnan(g.q[0, 170, 1]).all()) and bool(torch.isnan(g.v[0, :171, 1, 2]).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_rows_lose_no_digits(dtype):
    """A head that hardly forgets: the decay of a chunk is applied hundreds of times, and the states stay fp32's."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(28)
    length = 12345
    q, k, v = (r(1, length, 2, 64).to(dtype) for _ in range(3))
    ld = torch.tensor([-1e-5, -3e-4], device="cuda")
    _, last = Q.linear_attention_fwd(q, k, v, ld, 0.125)
    w = torch.exp(ld.double()[:, None] * torch.arange(length - 1, -1, -1, device="cuda"))
    want = torch.einsum("hl,blhi,blhj->bhij", w, k.double(), v.double())
    assert rel(last, want) <= 2e-6      # sums of 12345 products in 32 bits, chunk by chunk


def test_offsets_past_32_bits():
    from paper_2607_18020_b200 import sequence as Q
    r = gen(29)
    far = 1 << 32                                             # elements between the two rows
    big = torch.empty(far + 200 * 2 * 64, dtype=torch.bfloat16, device="cuda")
    q = torch.as_strided(big, (2, 200, 2, 64), (far, 128, 64, 1))
    q.copy_(r(2, 200, 2, 64))
    k, v = r(2, 200, 2, 64).bfloat16(), r(2, 200, 2, 64).bfloat16()
    ld = decays(2)
    o, _ = Q.linear_attention_fwd(q, k, v, ld)
    dense, _ = Q.linear_attention_fwd(q.contiguous(), k, v, ld)
    assert torch.equal(o, dense)
    o, _ = Q.linear_attention_fwd(k, q, v, ld)
    dense, _ = Q.linear_attention_fwd(k, q.contiguous(), v, ld)
    assert torch.equal(o, dense)


def test_streams_and_graphs():
    """On a stream of its own, and captured and replayed on new values, two calls in one graph."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(30)
    ts = [[r(1, 1500, 2, 64).bfloat16() for _ in range(4)] for _ in range(3)]
    ld, state = decays(2), r(1, 2, 64, 64)
    want = [(Q.linear_attention_fwd(*t[:3], ld, 0.1, state), Q.linear_attention_bwd(t[3], *t[:3], ld, 0.1, state)) for t in ts]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = Q.linear_attention_fwd(*ts[0][:3], ld, 0.1, state)
    side.synchronize()
    assert torch.equal(got[0], want[0][0][0]) and torch.equal(got[1], want[0][0][1])
    fixed = [[t.clone() for t in ts[i]] for i in range(2)]
    moving = state.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [(Q.linear_attention_fwd(*f[:3], ld, 0.1, state), Q.linear_attention_bwd(f[3], *f[:3], ld, 0.1, state)) for f in fixed]
        Q.linear_attention_step(moving, fixed[0][0][:, 0], fixed[0][1][:, 0], fixed[0][2][:, 0], ld, 0.1)
    for order in ((0, 1), (2, 0)):
        for f, i in zip(fixed, order):
            for a, b in zip(f, ts[i]):
                a.copy_(b)
        moving.copy_(state)
        graph.replay()
        torch.cuda.synchronize()
        for out, i in zip(outs, order):
            assert torch.equal(out[0][0], want[i][0][0]) and torch.equal(out[0][1], want[i][0][1])
            for a, b in zip(out[1], want[i][1]):
                assert torch.equal(a, b)
        one = state.clone()
        Q.linear_attention_step(one, *(ts[order[0]][j][:, 0] for j in range(3)), ld, 0.1)
        assert torch.equal(one, moving)


def test_autograd_and_values_only():
    from paper_2607_18020_b200 import sequence as Q
    r = gen(31)
    q, k, v = (r(1, 20, 2, 16).requires_grad_(True) for _ in range(3))
    ld = decays(2)
    state = r(1, 2, 16, 16)
    o, last = Q.linear_attention(q, k, v, ld, 0.5, state, return_state=True)
    last.sum().backward()                    # nothing asks for o
    _, _, want = wanted(q, k, v, ld, 0.5, state, torch.zeros_like(v), torch.ones_like(last))
    check_attention("gk", k.grad, want[1])
    assert float(q.grad.abs().sum()) == 0.0 and o.requires_grad
    with pytest.raises(ValueError, match="log_decay"):
        Q.linear_attention(q, k, v, ld.clone().requires_grad_(True))
    out = Q.linear_attention_step(state, q[:, 0], k[:, 0], v[:, 0], ld)
    with pytest.raises(RuntimeError, match="not differentiable"):
        out.sum().backward()
    kept = r(1, 2, 16, 16).requires_grad_(True)
    y = (kept * state).sum()
    with torch.no_grad():
        Q.linear_attention_step(state, q[:, 0], k[:, 0], v[:, 0], ld)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_refusals_of_the_python_layer():
    from paper_2607_18020_b200 import sequence as Q
    r = gen(32)
    q, k, v, ld = r(1, 9, 2, 16), r(1, 9, 2, 16), r(1, 9, 2, 8), decays(2)
    for bad in ((q, k[..., :8], v, ld), (q, k.half(), v, ld), (q, k, v[:, :5], ld), (q, k, v, ld[:1]), (q, k, v, ld.double()), (q[0], k, v, ld),
                (q, k, v[0], ld), (q.cpu(), k, v, ld), (q.double(), k, v, ld), (q, k.cpu(), v, ld)):
        with pytest.raises(ValueError):
            Q.linear_attention_fwd(*bad)
    with pytest.raises(ValueError):
        Q.linear_attention_fwd(q, k, v, ld, 1.0, r(1, 2, 8, 16))
    with pytest.raises(RuntimeError):
        Q.linear_attention_fwd(r(1, 4, 1, 129), r(1, 4, 1, 129), r(1, 4, 1, 8), ld[:1])
    with pytest.raises(RuntimeError):
        Q.linear_attention_fwd(q, k, v, ld, math.nan)
    with pytest.raises(ValueError):
        Q.linear_attention_step(r(1, 2, 8, 16).mT, q[:, 0], k[:, 0], v[:, 0], ld)
