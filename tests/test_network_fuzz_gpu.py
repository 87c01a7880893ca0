"""Randomly drawn sizes, strides, types and options (fixed seeds) of the sequence operators and the
orthogonalised update against the 64-bit forms, with guard bands around every output."""
import random

import pytest

torch = pytest.importorskip("torch")
from seq_util import ROUND, GuardedTorch, check, conv_ref, d64, ortho_ref, rel, scan_ref

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def draw(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def view(rng, gen, batch, length, channels, dtype):
    """An activation: dense, a slice of a wider one, or with its nodes ahead of its rows."""
    kind = rng.randrange(4)
    if kind == 0:
        return torch.randn(batch, length, channels, generator=gen, device="cuda").to(dtype)
    lead, tail = rng.randrange(5), rng.randrange(5)
    t = torch.randn(length if kind == 3 else batch, batch if kind == 3 else length, lead + channels + tail, generator=gen, device="cuda").to(dtype)
    t = t[..., lead:lead + channels]
    return t.transpose(0, 1) if kind == 3 else t


@pytest.mark.parametrize("seed", range(40))
def test_conv(seed, monkeypatch):
    from paper_2607_18020_b200 import sequence as Q
    guard = GuardedTorch()
    monkeypatch.setattr(Q, "torch", guard)
    rng, gen = random.Random(seed), torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, batch, length, channels, width = rng.choice(TYPES), draw(rng, 1, 6), draw(rng, 1, 700), draw(rng, 1, 300), rng.randrange(1, 5)
    x, gy = view(rng, gen, batch, length, channels, dtype), view(rng, gen, batch, length, channels, dtype)
    w = torch.randn(channels, width, generator=gen, device="cuda") * 0.5
    b = torch.randn(channels, generator=gen, device="cuda") if rng.random() < 0.7 else None
    s = torch.randn(batch, width - 1, channels, generator=gen, device="cuda").to(dtype) if rng.random() < 0.6 else None
    gs = torch.randn(batch, width - 1, channels, generator=gen, device="cuda").to(dtype) if rng.random() < 0.5 else None
    silu = rng.random() < 0.8
    y, left = Q.causal_conv_fwd(x, w, b, s, silu)
    g = Q.causal_conv_bwd(gy, x, w, b, s, silu, gs)
    leaves = [None if t is None else d64(t).requires_grad_(True) for t in (x, w, b, s)]
    ry, rleft = conv_ref(*leaves, silu)
    check("y", y, ry)
    assert torch.equal(left.double().cpu(), rleft.detach())
    total = (ry * d64(gy)).sum() + (0.0 if gs is None else (rleft * d64(gs)).sum())
    have = [(n, t) for n, t in zip(("x", "weight", "bias", "state"), leaves) if t is not None]
    for (n, t), e in zip(have, torch.autograd.grad(total, [t for _, t in have], allow_unused=True)):
        check("g" + n, getattr(g, n), torch.zeros_like(t) if e is None else e)
    torch.cuda.synchronize()
    guard.check()


@pytest.mark.parametrize("seed", range(60))
def test_scan(seed, monkeypatch):
    from paper_2607_18020_b200 import sequence as Q
    guard = GuardedTorch()
    monkeypatch.setattr(Q, "torch", guard)
    rng, gen = random.Random(1000 + seed), torch.Generator(device="cuda")
    gen.manual_seed(1000 + seed)
    dtype, batch, length, channels, n = rng.choice(TYPES), draw(rng, 1, 5), draw(rng, 1, 400), draw(rng, 1, 200), draw(rng, 1, 64)
    u, delta, B, C = (view(rng, gen, batch, length, k, dtype) for k in (channels, channels, n, n))
    go = view(rng, gen, batch, length, channels, dtype)
    z = view(rng, gen, batch, length, channels, dtype) if rng.random() < 0.7 else None
    A = -(0.2 + torch.rand(channels, n, generator=gen, device="cuda") * n)
    D = torch.randn(channels, generator=gen, device="cuda") if rng.random() < 0.7 else None
    bias = torch.randn(channels, generator=gen, device="cuda") - 2 if rng.random() < 0.7 else None
    s = torch.randn(batch, channels, n, generator=gen, device="cuda") if rng.random() < 0.6 else None
    gl = torch.randn(batch, channels, n, generator=gen, device="cuda") if rng.random() < 0.5 else None
    args = (u, delta, A, B, C, D, z, bias)
    out, last, kept = Q.selective_scan_fwd(*args, state=s, keep=True)
    g = Q.selective_scan_bwd(go, *args, state=s, kept=kept, gstate=gl)
    leaves = [None if t is None else d64(t).requires_grad_(True) for t in args + (s,)]
    rout, rlast = scan_ref(*leaves[:8], True, leaves[8])
    check("out", out, rout)
    check("state", last, rlast)
    total = (rout * d64(go)).sum() + (0.0 if gl is None else (rlast * d64(gl)).sum())
    names = ("u", "delta", "A", "B", "C", "D", "z", "delta_bias", "state")
    have = [(k, t) for k, t in zip(names, leaves) if t is not None]
    for (k, t), e in zip(have, torch.autograd.grad(total, [t for _, t in have], allow_unused=True)):
        check("g" + k, getattr(g, k), torch.zeros_like(t) if e is None else e)
    # the last node again, alone
    if length > 1:
        mid = Q.selective_scan_fwd(*(t if t is None or t.dim() < 3 else t[:, :-1] for t in args), state=s)[1]
        one = Q.selective_scan_step(mid, *(t if t is None or t.dim() < 3 else t[:, -1] for t in args))
        check("step", one, rout[:, -1])
        check("stepped state", mid, rlast)
    torch.cuda.synchronize()
    guard.check()


@pytest.mark.parametrize("seed", range(40))
def test_orthogonalize(seed, monkeypatch):
    from paper_2607_18020_b200 import binding, optim
    guard = GuardedTorch()
    monkeypatch.setattr(optim, "torch", guard)
    rng, gen = random.Random(2000 + seed), torch.Generator(device="cuda")
    gen.manual_seed(2000 + seed)
    dtype, rows, cols = rng.choice(TYPES), draw(rng, 1, 1500), draw(rng, 1, 1500)
    count = max(1, min(draw(rng, 1, 12), (1 << 23) // (rows * cols)))
    r = min(rows, cols) // 2 + 1
    g = torch.randn(count, rows, r, generator=gen, device="cuda") @ torch.randn(count, r, cols, generator=gen, device="cuda") / r ** 0.5
    g = (g + 0.3 * torch.randn(count, rows, cols, generator=gen, device="cuda")).to(dtype)
    x = optim.orthogonalize(g)
    want = ortho_ref(g.double(), 5, 1e-7)
    lim = 1.2e-4 if dtype == torch.float32 else 8.3e-3 + ROUND[dtype]
    for k in range(count):
        assert rel(x[k], want[k]) <= lim, (k, rel(x[k], want[k]))
    assert binding.diag_ortho_timeouts() == 0
    torch.cuda.synchronize()
    guard.check()
