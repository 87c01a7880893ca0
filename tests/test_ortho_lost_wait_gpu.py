"""A wait inside the orthogonalisation that nothing ends: it gives up, and the call's result says so."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
from test_optim_gpu import limit, matrices
from seq_util import d64, ortho_ref, rel

pytestmark = pytest.mark.gpu


def lost(g, steps=5):
    """fpde_diag_orthogonalize_lost on a stack of matrices."""
    from paper_2607_18020_b200 import binding
    out = torch.zeros_like(g)
    a = binding.OrthoArgs(dtype=binding.DTYPE_IDS[str(g.dtype)], steps=steps, count=g.shape[0], rows=g.shape[1], cols=g.shape[2],
                          grad=g.data_ptr(), grad_matrix=g.stride(0), grad_row=g.stride(1), out=out.data_ptr(), eps=1e-7)
    ws = torch.empty(max(1, binding.lib().fpde_orthogonalize_workspace_bytes(ctypes.byref(a))), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    binding.call_with("fpde_diag_orthogonalize_lost", a, 0)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("steps", [1, 5])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [(2, 40, 60), (1, 128, 256), (2, 300, 333), (1, 1100, 520)])
def test_the_result_is_nan_and_the_next_call_is_not(size, dtype, steps):
    from paper_2607_18020_b200 import binding, optim
    g = matrices(*size, dtype)
    assert bool(torch.isnan(lost(g, steps)).all())
    assert rel(optim.orthogonalize(g), ortho_ref(d64(g), 5, 1e-7)) <= limit(dtype)
    assert binding.diag_ortho_timeouts() == 0          # the wait lost on purpose does not count
