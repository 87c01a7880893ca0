"""The forms of the kernels that large calls take, against the 64-bit forms on the GPU (forms_util has the sizes, and
test_network_forms_host holds them to their forms).  Bounds: seq_util and test_optim_gpu."""
import pytest

torch = pytest.importorskip("torch")
from forms_util import CONV_LONG, CONV_STEP_ROWS, ORTHO, SCAN_TWO
from seq_util import GuardedTorch, ROUND, bound, conv_ref, ortho_ref, scan_ref
from test_optim_gpu import limit, matrices, muon_ref

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def g64(t):
    return None if t is None else t.detach().double()


def check(name, got, want):
    assert got.shape == want.shape
    r = float(torch.linalg.vector_norm(got.detach().double() - want) / torch.linalg.vector_norm(want))
    assert r <= bound(got.dtype), (name, r)


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


@pytest.mark.parametrize("view", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SCAN_TWO)
def test_scan(size, dtype, view, guard):
    """view: every activation one element into a wider one, so that rows start on odd elements."""
    from paper_2607_18020_b200 import sequence as Q
    batch, length, channels, n = size
    r = gen(channels + n)

    def act(k):
        return r(batch, length, k + 1).to(dtype)[..., 1:] if view else r(batch, length, k).to(dtype)
    u, delta, z, go, B, C = act(channels), act(channels), act(channels), act(channels), act(n), act(n)
    A = -(0.2 + torch.rand(channels, n, device="cuda") * n)
    D, bias, s, gl = r(channels), r(channels) - 2, r(batch, channels, n), r(batch, channels, n)
    args = (u, delta, A, B, C, D, z, bias)
    out, last, kept = Q.selective_scan_fwd(*args, state=s, keep=True)
    g = Q.selective_scan_bwd(go, *args, state=s, kept=kept, gstate=gl)
    leaves = [g64(t).requires_grad_(True) for t in args + (s,)]
    rout, rlast = scan_ref(*leaves[:8], True, leaves[8])
    check("out", out, rout.detach())
    check("state", last, rlast.detach())
    want = torch.autograd.grad([rout, rlast], leaves, [g64(go), g64(gl)])
    for k, e in zip(("u", "delta", "A", "B", "C", "D", "z", "delta_bias", "state"), want):
        check("g" + k, getattr(g, k), e)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", CONV_LONG)
def test_conv(size, dtype, guard):
    from paper_2607_18020_b200 import sequence as Q
    batch, length, channels, width, _ = size
    r = gen(channels)
    x, gy = r(batch, length, channels + 2).to(dtype)[..., 2:], r(batch, length, channels).to(dtype)
    w, b = 0.5 * r(channels, width), 0.5 * r(channels)
    s, gs = r(batch, width - 1, channels).to(dtype), r(batch, width - 1, channels).to(dtype)
    y, left = Q.causal_conv_fwd(x, w, b, s)
    g = Q.causal_conv_bwd(gy, x, w, b, s, True, gs)
    leaves = [g64(t).requires_grad_(True) for t in (x, w, b, s)]
    ry, rleft = conv_ref(*leaves, True)
    check("y", y, ry.detach())
    assert torch.equal(left.double(), rleft.detach())
    want = torch.autograd.grad([ry, rleft], leaves, [g64(gy), g64(gs)])
    for k, a, e in zip("xwbs", g, want):
        if e.numel():
            check("g" + k, a, e)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", CONV_STEP_ROWS)
def test_conv_step(size, dtype, guard):
    from paper_2607_18020_b200 import sequence as Q
    batch, channels = size
    r = gen(batch)
    x, w, b, window = r(batch, 3, channels).to(dtype), 0.5 * r(channels, 4), r(channels), r(batch, 3, channels).to(dtype)
    start = window.clone()
    ys = torch.stack([Q.causal_conv_step(x[:, t].contiguous(), window, w, b) for t in range(3)], 1)
    ry, rleft = conv_ref(g64(x), g64(w), g64(b), g64(start), True)
    check("y", ys, ry)
    assert torch.equal(window.double(), rleft)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", ORTHO)
def test_orthogonalize(size, dtype):
    from paper_2607_18020_b200 import binding, optim
    g = matrices(*size, dtype)
    x, want = optim.orthogonalize(g), ortho_ref(g.double(), 5, 1e-7)
    for k in range(size[0]):
        r = float(torch.linalg.vector_norm(x[k].double() - want[k]) / torch.linalg.vector_norm(want[k]))
        assert r <= limit(dtype), (k, r)
    assert torch.equal(x, optim.orthogonalize(g))
    assert binding.diag_ortho_timeouts() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(520, 264), (264, 520), (300, 301), (3, 301, 300), (2, 1000, 333), (768, 1536)])
def test_muon_step(shape, nesterov, dtype):
    from paper_2607_18020_b200 import optim
    full = (1,) * (3 - len(shape)) + shape
    w, g, m = (matrices(*full, t, seed=k).reshape(shape) for k, t in ((1, dtype), (2, dtype), (3, torch.float32)))
    before = g64(w)
    rw, rm = muon_ref(before, g64(g), g64(m), 0.1, 0.9, 0.05, nesterov)
    optim.muon_step(w, g, m, lr=0.1, momentum_decay=0.9, weight_decay=0.05, nesterov=nesterov)
    norm = torch.linalg.vector_norm
    assert norm(g64(m) - rm) <= 1e-6 * norm(rm)
    # the step is what the bound is about; a 16-bit weight also rounds, by its own size
    assert norm(g64(w) - rw) <= limit(dtype) * norm(rw - before) + ROUND[dtype] * norm(rw) + 1e-6 * norm(before)


def test_optimizer_on_a_large_parameter():
    """Muon over a parameter that leaves the one-SM form, and over one that does not, for three steps."""
    from paper_2607_18020_b200 import optim
    ws = [torch.nn.Parameter(matrices(1, r, c, torch.float32)[0]) for r, c in ((520, 264), (96, 64))]
    opt = optim.Muon(ws, lr=0.05, weight_decay=0.01)
    refs = [(g64(w), torch.zeros_like(w, dtype=torch.float64)) for w in ws]
    for k in range(3):
        for i, w in enumerate(ws):
            w.grad = matrices(1, *w.shape, torch.float32, seed=20 + k)[0]
            refs[i] = muon_ref(refs[i][0], g64(w.grad), refs[i][1], 0.05, 0.95, 0.01, True)
        opt.step()
    for w, (rw, rm) in zip(ws, refs):
        assert float((g64(w) - rw).norm() / rw.norm()) <= 3 * limit(torch.float32)
        assert float((opt.state[w]["momentum"].double() - rm).norm() / rm.norm()) <= 3e-6
