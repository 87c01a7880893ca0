"""Orthogonalised updates at the ends of the number range, against the 64-bit iteration (bounds: see test_optim_gpu)."""
import pytest

torch = pytest.importorskip("torch")
from seq_util import ROUND, d64, ortho_ref, rel
from test_optim_gpu import limit, matrices, muon_ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [1e-37, 1e-36, 1e-35, 1e-26, 1e34, 1e37])
@pytest.mark.parametrize("size", [(2, 40, 60), (1, 128, 256), (1, 300, 280), (2, 297, 333), (1, 520, 264)])
def test_any_scale(size, scale, dtype):
    """The entries are normal numbers of the type; their norm's reciprocal times 2^14 need not be.  Both forms of the call:
    matrices that stay on one SM and others, rows of a multiple of eight and others."""
    from paper_2607_18020_b200 import optim
    g = matrices(*size, dtype, scale=scale)
    assert bool(torch.isfinite(g).all())
    x = optim.orthogonalize(g, eps=0.0)
    assert rel(x, ortho_ref(d64(g), 5, 0.0)) <= limit(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [(4096, 2, 2), (16384, 3, 5), (4096, 5, 3), (4096, 4, 4), (2048, 8, 8), (1024, 8, 40), (512, 200, 8)])
def test_tiny_matrices_of_any_spectrum(size, dtype):
    """Every matrix of a large stack, among them almost singular ones.  Products of pairs leave 3.4445^5 2^-22 whatever the
    spectrum, and a 16-bit result rounds once more."""
    from paper_2607_18020_b200 import optim
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    m = torch.randn(*size, generator=g, device="cuda").to(dtype)
    x, want = optim.orthogonalize(m).double(), ortho_ref(m.double(), 5, 1e-7)
    error = torch.linalg.vector_norm(x - want, dim=(1, 2)) / torch.linalg.vector_norm(want, dim=(1, 2))
    assert float(error.max()) <= limit(torch.float32) + ROUND[dtype]


def test_values_but_no_gradient():
    from paper_2607_18020_b200 import optim
    g = matrices(1, 40, 60, torch.float32)[0]
    want = optim.orthogonalize(g)
    x = optim.orthogonalize(g.requires_grad_(True))
    assert torch.equal(x, want)
    with pytest.raises(RuntimeError, match="orthogonalize is not differentiable"):
        x.sum().backward()
    with torch.no_grad():
        assert not optim.orthogonalize(g).requires_grad


@pytest.mark.parametrize("shape", [(48, 80), (300, 264)])
def test_muon_step_of_tiny_gradients(shape):
    from paper_2607_18020_b200 import optim
    w, g, m = (matrices(1, *shape, torch.float32, scale=k, seed=i)[0] for i, k in enumerate((1.0, 1e-36, 1e-36)))
    rw, rm = muon_ref(d64(w), d64(g), d64(m), 0.1, 0.9, 0.0, True, eps=0.0)
    moved = torch.linalg.vector_norm(rw - d64(w))
    optim.muon_step(w, g, m, lr=0.1, momentum_decay=0.9, eps=0.0)
    assert rel(m, rm) <= 1e-6
    assert torch.linalg.vector_norm(d64(w) - rw) <= limit(torch.float32) * moved + 1e-6 * torch.linalg.vector_norm(rw)
