"""Rotation of heads by position and the norm before it, against the 64-bit form."""
import math

import pytest

torch = pytest.importorskip("torch")
from attention_util import norm_ref, rotary_ref
from seq_util import ROUND, GuardedTorch, check, d64

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


CASES = [  # batch, length, q heads, k heads, features, pairs, view, positions, offset
    (1, 1, 1, 1, 2, 1, "dense", None, 0), (2, 3, 2, 1, 1, 0, "dense", None, 0), (1, 5, 3, 0, 16, 8, "dense", None, 7),
    (2, 17, 4, 2, 44, 11, "dense", "rows", 0), (1, 100, 3, 3, 33, 16, "slice", None, 1000000), (3, 9, 5, 1, 64, 16, "slice", "rows", -3),
    (2, 33, 2, 2, 128, 64, "heads first", "shared", 0), (1, 65, 8, 2, 128, 32, "slice", None, 1 << 24), (1, 7, 1, 2, 255, 100, "odd", None, 5),
    (2, 40, 2, 2, 256, 128, "dense", "rows", 0), (1, 12, 2, 1, 96, 48, "odd", "shared", 2), (5, 1, 6, 2, 80, 40, "dense", "rows", 0),
    (1, 2600, 2, 1, 24, 12, "dense", None, 0), (1, 30, 1, 1, 130, 1, "dense", None, 0), (1, 30, 40, 8, 72, 36, "slice", None, 3),
    (0, 4, 2, 2, 8, 4, "dense", None, 0), (2, 0, 2, 2, 8, 4, "dense", None, 0), (2, 3, 0, 2, 8, 4, "dense", None, 0),
]


def heads(r, dtype, batch, length, n, dim, view):
    if view == "slice":
        return r(batch, length, n + 3, dim + 8).to(dtype)[:, :, 2:n + 2, 8:]
    if view == "odd":
        return r(batch, length, n, dim + 3).to(dtype)[..., 1:dim + 1]
    if view == "heads first":
        return r(batch, n, length, dim).to(dtype).transpose(1, 2)
    return r(batch, length, n, dim).to(dtype)


def inputs(case, dtype, seed=41):
    batch, length, hq, hk, dim, pairs, view, positions, offset = case
    r = gen(seed)
    q, gq = (heads(r, dtype, batch, length, hq, dim, view) for _ in range(2))
    k, gk = (heads(r, dtype, batch, length, hk, dim, view) if hk else None for _ in range(2))
    freq = (10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / max(1, pairs))).float()
    at = None
    if positions == "rows":
        at = torch.randint(-50, 5000, (batch, 2 * length), device="cuda")[:, ::2]
    if positions == "shared":
        at = torch.randint(0, 5000, (length,), device="cuda").expand(batch, length)
    return q, k, gq, gk, freq, {"positions": at, "offset": offset}


def cpu(how):
    return (None if how["positions"] is None else how["positions"].cpu(), how["offset"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_rotary(case, interleaved, dtype, guard):
    from paper_2607_18020_b200 import sequence as Q
    q, k, gq, gk, freq, how = inputs(case, dtype)
    got = Q.rotary_fwd(q, k, freq, interleaved=interleaved, **how)
    back = Q.rotary_bwd(gq, gk, freq, interleaved=interleaved, **how)
    for x, g, y, gx in ((q, gq, got[0], back[0]), (k, gk, got[1], back[1])):
        if x is None:
            assert y is None and gx is None
            continue
        leaf = d64(x).requires_grad_(True)
        want = rotary_ref(leaf, d64(freq), cpu(how)[0], how["offset"], interleaved)
        check("y", y, want)
        check("gx", gx, torch.autograd.grad(want, leaf, d64(g))[0])
        rest = slice(2 * freq.shape[0], None)
        assert torch.equal(y[..., rest], x[..., rest]) and torch.equal(gx[..., rest], g[..., rest])      # copied, not computed


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved,weights,eps", [(False, True, 1e-6), (True, True, 0.0), (False, False, 1e-2)])
@pytest.mark.parametrize("case", CASES)
def test_norm_rotary(case, interleaved, weights, eps, dtype, guard):
    from paper_2607_18020_b200 import sequence as Q
    q, k, gq, gk, freq, how = inputs(case, dtype, 42)
    dim, r = q.shape[3], gen(43)
    wq, wk = (1 + 0.2 * r(dim) for _ in range(2)) if weights else (None, None)
    wk = None if k is None else wk
    got = Q.norm_rotary_fwd(q, k, wq, wk, freq, interleaved=interleaved, eps=eps, **how)
    g = Q.norm_rotary_bwd(gq, gk, q, k, wq, wk, freq, interleaved=interleaved, eps=eps, **how)
    for x, up, w, y, gx, gw in ((q, gq, wq, got[0], g.q, g.q_weight), (k, gk, wk, got[1], g.k, g.k_weight)):
        if x is None:
            assert y is None and gx is None
            continue
        leaves = [d64(t).requires_grad_(True) for t in (x, w) if t is not None]
        want = rotary_ref(norm_ref(leaves[0], leaves[1] if weights else None, eps), d64(freq), cpu(how)[0], how["offset"], interleaved)
        check("y", y, want)
        for name, a, e in zip(("gx", "gw"), (gx, gw), torch.autograd.grad(want, leaves, d64(up))):
            if name == "gx" and dim == 1:
                # of a gradient along the head itself g r (1 - n^2) is left, with n^2 = 1 but for eps: the difference has the
                # rounding of its terms, of size |g r| <= |g / x|, and then that of the stored type, half a step of itself
                terms = float(d64(up).abs().max()) / float(d64(x).abs().min())
                assert bool(((a.double().cpu() - e).abs() <= 1e-5 * terms + ROUND[dtype] * e.abs()).all())
                continue
            check(name, a, e)


def test_norm_alone_and_its_gradient_by_differences():
    from paper_2607_18020_b200 import sequence as Q
    r = gen(44)
    x, w, up = r(2, 13, 3, 40), 1 + 0.1 * r(40), r(2, 13, 3, 40).double()

    def f(x, w):
        return (Q.norm_rotary(x, None, w)[0].double() * up).sum()
    leaves = [x.clone().requires_grad_(True), w.clone().requires_grad_(True)]
    check("norm", Q.norm_rotary(x, None, w)[0], norm_ref(d64(x), d64(w), 1e-6))
    h = 1e-2                                     # curvature h^2 = 1e-4 of the gradient's size, rounding 1e-7 / h
    for i, g in enumerate(torch.autograd.grad(f(*leaves), leaves)):
        d = r(*leaves[i].shape)
        hi, lo = ([t.detach() + s * h * d if j == i else t.detach() for j, t in enumerate(leaves)] for s in (1, -1))
        diff, along = float(f(*hi) - f(*lo)) / (2 * h), float((g.double() * d.double()).sum())
        scale = float(torch.linalg.vector_norm(g.double()) * torch.linalg.vector_norm(d.double()))
        assert abs(diff - along) <= 1e-3 * scale, (i, diff, along)


def test_autograd_of_both():
    from paper_2607_18020_b200 import sequence as Q
    r = gen(45)
    q, k, w = r(2, 9, 4, 32).requires_grad_(True), r(2, 9, 2, 32).requires_grad_(True), (1 + 0.1 * r(32)).requires_grad_(True)
    freq = Q.rotary_frequencies(16)
    a, b = Q.rotary(*Q.norm_rotary(q, k, w, None, freq, offset=3), freq, offset=-3)      # turned there and back
    up = r(2, 9, 4, 32)
    got = torch.autograd.grad(a, (q, w), up, retain_graph=True)                                              # nothing asks for k's
    lq, lw = d64(q).requires_grad_(True), d64(w).requires_grad_(True)
    want = rotary_ref(rotary_ref(norm_ref(lq, lw, 1e-6), d64(freq), None, 3, False), d64(freq), None, -3, False)
    check("y", a, want)
    for name, x, e in zip(("q", "w"), got, torch.autograd.grad(want, (lq, lw), d64(up))):
        check("g" + name, x, e)
    assert float(torch.autograd.grad(b.sum(), k)[0].abs().sum()) > 0
    with pytest.raises(ValueError, match="inv_freq"):
        Q.rotary(q, k, freq.clone().requires_grad_(True))


def test_relative_positions_are_all_that_counts():
    """q.k of two nodes depends on the distance between them, far along the row as well."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(46)
    q, k, freq = r(1, 1, 1, 64), r(1, 1, 1, 64), Q.rotary_frequencies(32)
    near = (Q.rotary(q, None, freq, offset=20)[0] * Q.rotary(k, None, freq, offset=11)[0]).sum()
    far = (Q.rotary(q, None, freq, offset=20 + (1 << 27))[0] * Q.rotary(k, None, freq, offset=11 + (1 << 27))[0]).sum()
    size = float(torch.linalg.vector_norm(q) * torch.linalg.vector_norm(k))
    assert abs(float(near - far)) <= 1e-6 * size      # angles to 2^27 * 2^-53, cosines and products to 2^-23


def test_frequencies():
    from paper_2607_18020_b200 import sequence as Q
    plain = Q.rotary_frequencies(32, device="cpu")
    assert torch.allclose(plain.double(), 10000.0 ** (-torch.arange(32).double() / 32), rtol=2 ** -23)
    assert torch.allclose(Q.rotary_frequencies(32, stretch=4.0, device="cpu"), plain / 4)
    parts = Q.rotary_frequencies(32, stretch=4.0, length=2048, device="cpu")
    turns = 2048 * plain / (2 * math.pi)
    assert torch.equal(parts[turns > 32], plain[turns > 32]) and torch.allclose(parts[turns < 1], plain[turns < 1] / 4)
    assert bool((parts <= plain).all()) and bool((parts >= plain / 4 * (1 - 1e-6)).all())
    with pytest.raises(ValueError):
        Q.rotary_frequencies(0)


def test_nan_and_infinity_stay_in_their_head():
    from paper_2607_18020_b200 import sequence as Q
    r = gen(47)
    q, freq, w = r(1, 20, 3, 32), Q.rotary_frequencies(16), r(32)
    clean, turned = Q.norm_rotary_fwd(q, None, w, None, freq)[0], Q.rotary_fwd(q, None, freq)[0]
    q[0, 5, 1, 3], q[0, 9, 2, 20] = float("nan"), float("inf")
    y, z = Q.norm_rotary_fwd(q, None, w, None, freq)[0], Q.rotary_fwd(q, None, freq)[0]
    same = torch.ones(1, 20, 3, dtype=torch.bool, device="cuda")
    same[0, 5, 1] = same[0, 9, 2] = False
    assert torch.equal(y[same], clean[same]) and bool(torch.isnan(y[0, 5, 1]).all())
    others = torch.ones_like(z, dtype=torch.bool)
    others[0, 5, 1, [3, 19]] = False
    others[0, 9, 2, [4, 20]] = False
    assert torch.equal(z[others], turned[others]) and not bool(torch.isfinite(z[~others]).any())


def test_offsets_past_32_bits_and_graph():
    from paper_2607_18020_b200 import sequence as Q
    r = gen(48)
    far = 1 << 32
    big = torch.empty(far + 2048, dtype=torch.bfloat16, device="cuda")
    q = torch.as_strided(big, (2, 8, 2, 64), (far, 128, 64, 1))
    q.copy_(r(2, 8, 2, 64))
    at = torch.arange(8, device="cuda").expand(2, 8).contiguous()
    freq = Q.rotary_frequencies(32)
    assert torch.equal(Q.rotary_fwd(q, None, freq, at)[0], Q.rotary_fwd(q.contiguous(), None, freq)[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = Q.norm_rotary_fwd(q, None, None, None, freq, at)
        g = Q.norm_rotary_bwd(q, None, q, None, None, None, freq, at)
    at += 11                                 # positions are read when the graph runs
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, Q.norm_rotary_fwd(q, None, None, None, freq, offset=11)[0])
    assert torch.equal(g.q, Q.norm_rotary_bwd(q, None, q, None, None, None, freq, offset=11).q)


def test_refusals_of_the_python_layer():
    from paper_2607_18020_b200 import sequence as Q
    r = gen(49)
    q, k, freq = r(1, 9, 2, 16), r(1, 9, 1, 16), Q.rotary_frequencies(8)
    for bad in ((q[0], k, freq), (q, k[0], freq), (q, k[..., :8], freq), (q, k[:, :5], freq), (q, k.half(), freq), (q.cpu(), k, freq), (q, k.cpu(), freq),
                (q, k, freq.double()), (q, k, freq.cpu()), (q, k, Q.rotary_frequencies(9)), (q, k, freq[None])):
        with pytest.raises(ValueError):
            Q.rotary_fwd(*bad)
    for at in (torch.zeros(1, 8, dtype=torch.int64, device="cuda"), torch.zeros(1, 9, device="cuda"), torch.zeros(1, 9, dtype=torch.int64)):
        with pytest.raises(ValueError):
            Q.rotary_fwd(q, k, freq, at)
    with pytest.raises(ValueError):
        Q.norm_rotary_fwd(q, k, r(8))
    with pytest.raises(ValueError):
        Q.norm_rotary_bwd(q, None, q, k)
    with pytest.raises(RuntimeError):
        Q.norm_rotary_fwd(q, k, eps=-1.0)
    with pytest.raises(RuntimeError):
        Q.rotary_fwd(r(1, 2, 1, 257), None, freq)
