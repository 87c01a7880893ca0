"""The example that runs the sequence operators, the residual loss and the optimiser together."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_march_burgers_learns_and_marches():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "march_burgers.py")
    spec = importlib.util.spec_from_file_location("march_burgers", path)
    M = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(M)
    net, losses, x, t = M.train(nx=64, nt=33, steps=60, width=32)
    assert all(v == v for v in losses)
    assert min(losses[-5:]) < 0.5 * losses[0], (losses[0], losses[-5:])
    with torch.no_grad():
        whole = net(x, t)
    # the same sums in another order, through 2 layers and 33 nodes of fp32
    assert float((whole - net.march(x, t)).abs().max()) <= 1e-3 * float(whole.abs().max())
