"""Linear attention in every form of its kernels, and rotation, norms and attention together as a mixer uses them: prompts
and steps, gradients through all of it, graphs, streams, drawn sizes."""
import random

import pytest

torch = pytest.importorskip("torch")
from attention_forms import MIXED, ONE, PIECES, PLAIN
from attention_util import attention_bound, check_attention, linear_ref, norm_ref, rotary_ref
from seq_util import GuardedTorch, d64, rel

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


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


@pytest.fixture(autouse=True)
def no_wait_gives_up():
    from paper_2607_18020_b200 import binding
    before = binding.diag_linear_timeouts()
    yield
    torch.cuda.synchronize()
    assert binding.diag_linear_timeouts() == before


def decays(heads):
    return torch.tensor([(-0.004, -0.2, 0.0)[i % 3] for i in range(heads)], device="cuda")


def both_passes(q, k, v, ld, scale, s, go, gs):
    """o, the last state and the gradients against the 64-bit form's."""
    from paper_2607_18020_b200 import sequence as Q
    o, last = Q.linear_attention_fwd(q, k, v, ld, scale, s)
    g = Q.linear_attention_bwd(go, q, k, v, ld, scale, s, gs)
    leaves = [t.requires_grad_(True) for t in map(d64, (q, k, v, s)) if t is not None]
    ro, rlast = linear_ref(*leaves[:3], d64(ld), scale, leaves[3] if s is not None else None)
    loss = (ro * d64(go)).sum() if gs is None else (ro * d64(go)).sum() + (rlast * d64(gs)).sum()
    want = torch.autograd.grad(loss, leaves)
    check_attention("o", o, ro.detach())
    check_attention("state", last, rlast.detach())
    for name, a, e in zip(("gq", "gk", "gv", "gstate"), [t for t in g if t is not None], want):
        check_attention(name, a, e)


@pytest.mark.parametrize("ends", ["states", "no states"])
@pytest.mark.parametrize("case", PIECES + ONE)
def test_forms_on_tensor_cores(case, ends, guard):
    batch, length, heads, dk, dv = case
    r = gen(41)
    pad = [-n % 8 for n in (dk, dv)]         # rows of whole 16 bytes, as TMA reads them
    q, k = (r(batch, length, heads, dk + pad[0]).to(BF16)[..., :dk] for _ in range(2))
    v, go = (r(batch, length, heads, dv + pad[1]).to(BF16)[..., :dv] for _ in range(2))
    s, gs = (r(batch, heads, dk, dv) for _ in range(2)) if ends == "states" else (None, None)
    both_passes(q, k, v, decays(heads), dk ** -0.5, s, go, gs)


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("case", PLAIN + MIXED)
def test_forms_of_32_bit_arithmetic(case, dtype, guard):
    batch, length, heads, dk, dv = case
    r = gen(42)
    q, k, v, go = (r(batch, length, heads, n).to(dtype) for n in (dk, dk, dv, dv))
    both_passes(q, k, v, decays(heads), dk ** -0.5, r(batch, heads, dk, dv), go, r(batch, heads, dk, dv))


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("case", [PIECES[0], PIECES[6], PIECES[4]])
def test_one_array_that_tma_cannot_read(case, which, guard):
    """Its marches take the other form, the rest the tensor cores; gk still starts from the states that gv's march has joined."""
    batch, length, heads, dk, dv = case
    r = gen(43)
    t = [r(batch, length, heads, n).to(BF16) for n in (dk, dk, dv, dv)]
    odd = r(batch, length, heads, t[which].shape[3] + 1).to(BF16)[..., 1:]
    t[which] = odd
    both_passes(*t[:3], decays(heads), dk ** -0.5, r(batch, heads, dk, dv), t[3], r(batch, heads, dk, dv))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_head_for_all_and_repeated_rows_in_pieces(dtype):
    """Keys with a head stride of zero, values with a batch stride of zero, queries that are the keys themselves."""
    r = gen(44)
    k = r(2, 1000, 1, 64).to(dtype).expand(2, 1000, 3, 64)
    v, go = r(1, 1000, 3, 40).to(dtype).expand(2, 1000, 3, 40), r(2, 1000, 3, 40).to(dtype)
    both_passes(k, k, v, decays(3), 0.1, None, go, None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dims", [(64, 64), (128, 72), (32, 128)])
def test_infinities_and_nan_in_rows_of_pieces(dims, dtype):
    """A node reaches no earlier one in any piece, and every later one that its product enters."""
    from paper_2607_18020_b200 import sequence as Q
    dk, dv = dims
    r = gen(45)
    q, k, v, go = (r(1, 1000, 1, n).to(dtype) for n in (dk, dk, dv, dv))
    ld = torch.zeros(1, device="cuda")
    clean, cg = Q.linear_attention_fwd(q, k, v, ld, 0.1)[0], Q.linear_attention_bwd(go, q, k, v, ld, 0.1)
    for at in (0, 127, 128, 400, 640, 999):
        bad = v.clone()
        bad[0, at, 0, 3] = float("nan")
        o, last = Q.linear_attention_fwd(q, k, bad, ld, 0.1)
        assert torch.equal(o[:, :at], clean[:, :at]) and torch.equal(o[..., :3], clean[..., :3])
        assert bool(torch.isnan(o[:, at:, :, 3]).all()) and bool(torch.isnan(last[..., 3]).all())
        bad = go.clone()
        bad[0, at, 0, 3] = float("inf")
        g = Q.linear_attention_bwd(bad, q, k, v, ld, 0.1)
        assert torch.equal(g.q[:, :at], cg.q[:, :at]) and torch.equal(g.q[:, at + 1:], cg.q[:, at + 1:])
        assert torch.equal(g.k[:, at + 1:], cg.k[:, at + 1:]) and torch.equal(g.v[:, at + 1:], cg.v[:, at + 1:])
        assert not bool(torch.isfinite(g.q[:, at]).any()) and not bool(torch.isfinite(g.k[:, :at + 1]).any())
        assert not bool(torch.isfinite(g.v[:, :at + 1, :, 3]).any()) and torch.equal(g.v[..., 4:], cg.v[..., 4:])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_decays_of_every_size_in_pieces(dtype):
    """From one that forgets everything within a node to one that never does, and a state that grows."""
    r = gen(46)
    ld = torch.tensor([-float("inf"), -100.0, -3.0, -1e-3, 0.0, 2e-3], device="cuda")
    q, k, v, go = (r(1, 700, 6, 64).to(dtype) for _ in range(4))
    both_passes(q, k, v, ld, 0.125, r(1, 6, 64, 64), go, r(1, 6, 64, 64))


@pytest.mark.parametrize("seed", range(16))
def test_drawn_sizes(seed, guard):
    rnd = random.Random(seed)
    r = gen(100 + seed)
    dtype = (F32, BF16, BF16, F16)[seed % 4]
    batch, heads, dk, dv = rnd.randint(1, 3), rnd.randint(1, 4), rnd.randint(1, 128), rnd.randint(1, 128)
    length = rnd.choice((rnd.randint(1, 64), rnd.randint(65, 300), rnd.randint(300, 900)))

    def view(n):
        lead, tail = rnd.choice(((0, 0), (8, 8), (1, 2))), rnd.randint(0, 1)
        x = r(batch, length + tail, heads + tail, n + sum(lead)).to(dtype)
        return x[:, tail:, tail:, lead[0]:lead[0] + n]
    q, k, v, go = (view(n) for n in (dk, dk, dv, dv))
    s, gs = (r(batch, heads, dk, dv) if rnd.random() < 0.5 else None for _ in range(2))
    both_passes(q, k, v, decays(heads), rnd.uniform(0.05, 1.0), s, go, gs)


# ------------------------------------------------------------------------------------- the operators together
def mixer(Q, x, heads, dk, dv, weights, freq, ld, offset=0, state=None):
    """A layer's mixer: queries, keys and values side by side in x, queries and keys normed and turned, the attention's heads normed."""
    b, n, _ = x.shape
    q, k, v = torch.split(x, [heads * dk, heads * dk, heads * dv], -1)
    q, k = Q.norm_rotary(q.unflatten(-1, (heads, dk)), k.unflatten(-1, (heads, dk)), weights[0], weights[1], freq, offset=offset)
    if n == 1 and state is not None:
        o = Q.linear_attention_step(state, q[:, 0], k[:, 0], v.unflatten(-1, (heads, dv))[:, 0], ld, dk ** -0.5)[:, None]
    else:
        o, state = Q.linear_attention(q, k, v.unflatten(-1, (heads, dv)), ld, dk ** -0.5, state, True)
    return Q.norm_rotary(o, None, weights[2], None, None)[0], state


def mixer_ref(x, heads, dk, dv, weights, freq, ld):
    q, k, v = torch.split(x, [heads * dk, heads * dk, heads * dv], -1)
    q, k = (rotary_ref(norm_ref(t.unflatten(-1, (heads, dk)), w, 1e-6), freq, None, 0, False) for t, w in ((q, weights[0]), (k, weights[1])))
    o, last = linear_ref(q, k, v.unflatten(-1, (heads, dv)), ld, dk ** -0.5, None)
    return norm_ref(o, weights[2], 1e-6), last


def mixer_inputs(dtype, seed, batch, length, heads, dk, dv):
    from paper_2607_18020_b200 import sequence as Q
    r = gen(seed)
    x = r(batch, length, heads * (2 * dk + dv)).to(dtype)
    w = [1 + 0.2 * r(n) for n in (dk, dk, dv)]
    return x, w, Q.rotary_frequencies(dk // 2, device="cuda"), decays(heads), r(batch, length, heads, dv).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("sizes", [(2, 50, 3, 16, 24), (1, 700, 2, 64, 64), (1, 300, 1, 128, 128)])
def test_mixer_and_its_gradients(sizes, dtype):
    """Four roundings to the type follow one another (norm and rotation, attention, norm, each within its own bound), and a norm
    takes errors on at their relative size; backwards as many again: three and six bounds."""
    from paper_2607_18020_b200 import sequence as Q
    x, w, freq, ld, go = mixer_inputs(dtype, 51, *sizes)
    leaves = [t.requires_grad_(True) for t in (x, *w)]
    o, _ = mixer(Q, x, *sizes[2:], w, freq, ld)
    grads = torch.autograd.grad(o, leaves, go)
    ref = [d64(t).requires_grad_(True) for t in leaves]
    ro, _ = mixer_ref(ref[0], *sizes[2:], ref[1:], d64(freq), d64(ld))
    want = torch.autograd.grad(ro, ref, d64(go))
    assert rel(o, ro.detach()) <= 3 * attention_bound(dtype)
    for g, e in zip(grads, want):
        assert rel(g, e) <= 6 * attention_bound(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_mixer_steps_agree_with_a_prompt(dtype):
    """A prompt, then one node after the other, against all at once in 64 bits."""
    from paper_2607_18020_b200 import sequence as Q
    sizes = (2, 170, 2, 64, 48)
    x, w, freq, ld, _ = mixer_inputs(dtype, 52, *sizes)
    with torch.no_grad():
        o, state = mixer(Q, x[:, :160], *sizes[2:], w, freq, ld)
        outs = [o]
        for t in range(160, 170):
            outs.append(mixer(Q, x[:, t:t + 1], *sizes[2:], w, freq, ld, t, state)[0])
    ro, rlast = mixer_ref(d64(x), *sizes[2:], [d64(t) for t in w], d64(freq), d64(ld))
    got = torch.cat(outs, 1)
    assert rel(got, ro) <= 3 * attention_bound(dtype) and rel(got[:, 160:], ro[:, 160:]) <= 3 * attention_bound(dtype)
    assert rel(state, rlast) <= 2 * attention_bound(dtype)        # keys rounded to the type


def test_mixer_gradients_against_differences():
    """Central differences of the 32-bit mixer along a direction, step 1e-2 of the inputs' size: an error of third order,
    1e-4 times a few, and rounding of 1e-6 / 1e-2; held to 3e-3 of the product of the norms."""
    from paper_2607_18020_b200 import sequence as Q
    sizes = (1, 40, 2, 16, 16)
    x, w, freq, ld, go = mixer_inputs(F32, 53, *sizes)
    leaves = [t.clone().requires_grad_(True) for t in (x, *w)]
    f = lambda ts: (mixer(Q, ts[0], *sizes[2:], ts[1:], freq, ld)[0].double() * go.double()).sum()
    grads = torch.autograd.grad(f(leaves), leaves)
    r = gen(54)
    for i, g in enumerate(grads):
        d = r(*g.shape)
        with torch.no_grad():
            hi, lo = ([t + s * 1e-2 * d if j == i else t for j, t in enumerate(leaves)] for s in (1, -1))
            diff = float(f(hi) - f(lo)) / 2e-2
        along = float((g.double() * d.double()).sum())
        assert abs(diff - along) <= 3e-3 * float(g.double().norm() * d.double().norm()), (i, diff, along)


def test_mixer_captured_forwards_and_backwards():
    """Training of the mixer in a graph, with the gradients in place, against the same calls one by one, on new values."""
    from paper_2607_18020_b200 import sequence as Q
    sizes = (1, 600, 2, 64, 64)
    x, w, freq, ld, go = mixer_inputs(BF16, 55, *sizes)
    leaves = [t.requires_grad_(True) for t in (x, *w)]

    def step():
        o, _ = mixer(Q, leaves[0], *sizes[2:], leaves[1:], freq, ld)
        return [o.detach(), *torch.autograd.grad(o, leaves, go)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    r = gen(56)
    for _ in range(2):
        with torch.no_grad():
            x.copy_(r(*x.shape))
            go.copy_(r(*go.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for a, e in zip(got, step()):
            assert torch.equal(a, e)


def test_two_streams_at_once():
    """Calls on two streams share no workspace: each gives the bits that it gives alone."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(57)
    sets = [[r(1, 4096, 2, 64).bfloat16() for _ in range(4)] for _ in range(2)]
    ld = decays(2)
    call = lambda t: [*Q.linear_attention_fwd(*t[:3], ld, 0.1), *Q.linear_attention_bwd(t[3], *t[:3], ld, 0.1)[:3]]
    want = [call(t) for t in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(call(sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, e) for a, e in zip(g, want[i]))


def test_only_the_gradients_that_are_asked_for():
    """A state without a gradient, none wanted of the values, and a last state that nobody takes leave the others as they are."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(58)
    ld = decays(2)
    for dtype, length in ((F32, 70), (BF16, 700)):
        q, k, v, go = (r(1, length, 2, 64).to(dtype) for _ in range(4))
        s, gs = r(1, 2, 64, 64), r(1, 2, 64, 64)
        want = Q.linear_attention_bwd(go, q, k, v, ld, 0.1, s, gs)
        leaves = [q.clone().requires_grad_(True), k.clone().requires_grad_(True), v, s]
        o, last = Q.linear_attention(leaves[0], leaves[1], v, ld, 0.1, s, return_state=True)
        gq, gk = torch.autograd.grad([o, last], leaves[:2], [go, gs])
        assert torch.equal(gq, want.q)
        # gk starts from the joined states of gv's march, which keeps 16 bits of b's weights instead of 24 where no state leaves.  That
        # moves a state by 2^-17 of itself at most, and so the bf16 factor made of it by one step of 2^-7 in no more than 2^-9 of its
        # elements: 2^-11.5 in the 2-norm.  With the two results' own roundings, 2^-9 each way: within 2^-8 + 2^-11.5 < 2^-7.
        assert rel(gk, want.k) <= (2.0 ** -7 if dtype == BF16 else 0.0)
        o2 = Q.linear_attention(q.requires_grad_(True), k, v, ld, 0.1, s)
        check_attention("o", o2.detach(), o.detach().double())
        (gq,) = torch.autograd.grad(o2, [q], go)
        assert torch.equal(gq, want.q)
        q.requires_grad_(False)
