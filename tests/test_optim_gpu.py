"""Orthogonalised updates against the 64-bit iteration.

Bounds (relative 2-norm), from the iteration itself: a step multiplies what rounding left in the smallest
singular directions by at most a = 3.4445, five of them by 485.  fp32 matrices are multiplied as pairs with
22 bits, so an error of 485 * 2^-22 = 1.2e-4 can be left; 16-bit ones with 11 bits per factor, where each of
the five steps adds at most (|b| + |c|) 2^-12 of rounded factors, 5 * 6.81 * 2^-12 = 8.3e-3, and the output's
own rounding."""
import pytest

torch = pytest.importorskip("torch")
from seq_util import ROUND, GuardedTorch, d64, ortho_ref, rel

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def limit(dtype):
    return 1.2e-4 if dtype == torch.float32 else 8.3e-3 + ROUND[dtype]


def matrices(count, rows, cols, dtype, scale=1e-2, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = min(rows, cols) // 2 + 1
    a = torch.randn(count, rows, r, generator=g, device="cuda") @ torch.randn(count, r, cols, generator=g, device="cuda")
    return ((a / r ** 0.5 + 0.3 * torch.randn(count, rows, cols, generator=g, device="cuda")) * scale).to(dtype)


SIZES = [(1, 1, 1), (1, 1, 7), (1, 7, 1), (2, 5, 3), (3, 16, 16), (2, 33, 65), (1, 128, 128), (2, 129, 127), (1, 64, 300),
         (1, 300, 64), (1, 256, 512), (2, 260, 390), (1, 500, 131), (1, 640, 640), (5, 96, 200)]


@pytest.fixture
def guard(monkeypatch):
    from paper_2607_18020_b200 import optim
    g = GuardedTorch()
    monkeypatch.setattr(optim, "torch", g)
    yield g
    torch.cuda.synchronize()
    g.check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_orthogonalize(size, dtype, guard):
    from paper_2607_18020_b200 import binding, optim
    g = matrices(*size, dtype)
    x = optim.orthogonalize(g)
    r = rel(x, ortho_ref(d64(g), 5, 1e-7))
    assert r <= limit(dtype), r
    assert binding.diag_ortho_timeouts() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(8, 1000, 1030), (3, 1500, 700), (1, 2300, 2100), (20, 257, 513), (1, 33, 70001),
                                  (1, 30000, 200)])
def test_orthogonalize_large(size, dtype, guard):
    """Sizes that fill the GPU; the 64-bit form runs on it too."""
    from paper_2607_18020_b200 import binding, optim
    g = matrices(*size, dtype)
    x = optim.orthogonalize(g)
    assert rel(x, ortho_ref(g.double(), 5, 1e-7)) <= limit(dtype)
    assert binding.diag_ortho_timeouts() == 0


@pytest.mark.parametrize("steps", [0, 1, 2, 7])
def test_number_of_steps(steps):
    from paper_2607_18020_b200 import optim
    g = matrices(2, 70, 90, torch.float32)
    assert rel(optim.orthogonalize(g, steps=steps), ortho_ref(d64(g), steps, 1e-7)) <= limit(torch.float32)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1.0, 1e25])
def test_scales(scale):
    from paper_2607_18020_b200 import optim
    g = matrices(1, 40, 60, torch.float32, scale=scale)
    assert rel(optim.orthogonalize(g, eps=0.0), ortho_ref(d64(g), 5, 0.0)) <= limit(torch.float32)


def test_zero_matrix_gives_zero_and_spoils_no_other():
    from paper_2607_18020_b200 import optim
    g = matrices(3, 40, 60, torch.float32)
    alone = optim.orthogonalize(g[2])
    g[1] = 0
    x = optim.orthogonalize(g)
    assert bool((x[1] == 0).all()) and torch.equal(x[2], alone)
    g[1, 3, 3] = float("nan")
    x = optim.orthogonalize(g)
    assert bool(torch.isnan(x[1]).all()) and torch.equal(x[2], alone)


def test_strided_matrices():
    from paper_2607_18020_b200 import optim
    whole = matrices(2, 50, 121, torch.float32)
    part = whole[:, 3:43, 7:77]
    assert torch.equal(optim.orthogonalize(part), optim.orthogonalize(part.contiguous()))
    t = part.transpose(1, 2)
    assert torch.equal(optim.orthogonalize(t), optim.orthogonalize(t.contiguous()))


def test_empty():
    from paper_2607_18020_b200 import optim
    for shape in ((0, 4, 5), (2, 0, 5), (2, 4, 0)):
        assert optim.orthogonalize(torch.empty(shape, device="cuda")).shape == shape


def muon_ref(w, g, m, lr, mu, wd, nesterov, steps=5, eps=1e-7):
    m = mu * m + g
    u = g + mu * m if nesterov else m
    o = ortho_ref(u, steps, eps)
    return (1 - lr * wd) * w - lr * max(1.0, w.shape[-2] / w.shape[-1]) ** 0.5 * o, m


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(48, 80), (80, 48), (3, 100, 37)])
def test_muon_step(shape, nesterov, dtype):
    from paper_2607_18020_b200 import optim
    full = (1,) * (3 - len(shape)) + shape
    w, g, m = (matrices(*full, t, seed=k).reshape(shape) for k, t in ((1, dtype), (2, dtype), (3, torch.float32)))
    rw, rm = muon_ref(d64(w), d64(g), d64(m), 0.1, 0.9, 0.05, nesterov)
    moved = rw - d64(w)
    before = d64(w)
    optim.muon_step(w, g, m, lr=0.1, momentum_decay=0.9, weight_decay=0.05, nesterov=nesterov)
    assert rel(m, rm) <= 1e-6
    # the step is what the bound is about; a 16-bit weight also rounds, by its own size
    err = torch.linalg.vector_norm(d64(w) - rw)
    assert err <= limit(dtype) * torch.linalg.vector_norm(moved) + ROUND[dtype] * torch.linalg.vector_norm(rw) + 1e-6 * torch.linalg.vector_norm(before)


def test_optimizer_class_and_its_state():
    from paper_2607_18020_b200 import optim
    w = torch.nn.Parameter(matrices(1, 40, 24, torch.bfloat16)[0])
    opt = optim.Muon([w], lr=0.05, weight_decay=0.01)
    rw, rm = d64(w), torch.zeros(40, 24, dtype=torch.float64)
    for k in range(3):
        w.grad = matrices(1, 40, 24, torch.bfloat16, seed=20 + k)[0]
        rw, rm = muon_ref(rw, d64(w.grad), rm, 0.05, 0.95, 0.01, True)
        opt.step()
    assert rel(w, rw) <= 3 * (limit(torch.bfloat16) + ROUND[torch.bfloat16])
    other = optim.Muon([torch.nn.Parameter(w.detach().clone())])
    other.load_state_dict(opt.state_dict())
    got = next(iter(other.state.values()))["momentum"]
    assert got.dtype == torch.float32 and torch.equal(got, opt.state[w]["momentum"])


def test_refusals():
    from paper_2607_18020_b200 import optim
    from paper_2607_18020_b200.binding import FpdeError
    g = matrices(1, 8, 8, torch.float32)[0]
    with pytest.raises(ValueError):
        optim.orthogonalize(g.cpu())
    with pytest.raises(ValueError):
        optim.orthogonalize(g[0])
    with pytest.raises(ValueError):
        optim.orthogonalize(g.double())
    with pytest.raises(FpdeError):
        optim.orthogonalize(g, steps=-1)
    with pytest.raises(FpdeError):
        optim.orthogonalize(g, eps=float("nan"))
    with pytest.raises(ValueError):
        optim.muon_step(g, g, g.half(), lr=0.1)
    with pytest.raises(ValueError):
        optim.muon_step(g.t(), g, g.clone(), lr=0.1)
    with pytest.raises(ValueError):
        optim.muon_step(g, g[:4], g.clone(), lr=0.1)
    with pytest.raises(ValueError):
        optim.Muon([torch.nn.Parameter(torch.zeros(4, device="cuda"))])
