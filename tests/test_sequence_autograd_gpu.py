"""How the sequence operators behave towards autograd beyond their gradients: tensors that single-node calls move
on in place, and results that have no gradient."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def randn(*s, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*s, generator=g, device="cuda")


def conv_step_args():
    return randn(2, 8), randn(2, 3, 8), randn(8, 4), randn(8)


def scan_step_args():
    c, n = 8, 16
    return randn(2, c, n), randn(2, c), randn(2, c), -torch.rand(c, n, device="cuda"), randn(2, n), randn(2, n)


def test_a_window_moved_on_is_not_taken_for_the_one_saved():
    from paper_2607_18020_b200 import sequence as Q
    x1, window, w, b = conv_step_args()
    w.requires_grad_(True)
    y = Q.causal_conv(randn(2, 5, 8), w, b, state=window)
    with torch.no_grad():
        Q.causal_conv_step(x1, window, w, b)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_a_state_moved_on_is_not_taken_for_the_one_saved():
    from paper_2607_18020_b200 import sequence as Q
    state, u, delta, A, B, C = scan_step_args()
    A.requires_grad_(True)
    rows = [t[:, None].expand(-1, 5, -1) for t in (u, delta)] + [A] + [t[:, None].expand(-1, 5, -1) for t in (B, C)]
    y = Q.selective_scan(*rows, state=state)
    with torch.no_grad():
        Q.selective_scan_step(state, u, delta, A, B, C)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_steps_count_as_changes_in_every_mode():
    from paper_2607_18020_b200 import sequence as Q
    x, window, w, b = conv_step_args()
    state, *rest = scan_step_args()
    for _ in range(2):
        before = window._version, state._version
        Q.causal_conv_step(x, window, w, b)
        Q.selective_scan_step(state, *rest)
        assert window._version > before[0] and state._version > before[1]
    with torch.inference_mode():
        window, state = window.clone(), state.clone()      # these carry no count, and need none
        Q.causal_conv_step(x, window, w, b)
        Q.selective_scan_step(state, *rest)


@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_conv_step_has_values_but_no_gradient(which):
    from paper_2607_18020_b200 import sequence as Q
    args = conv_step_args()
    want = Q.causal_conv_step(args[0], args[1].clone(), *args[2:])
    args[which].requires_grad_(True)
    y = Q.causal_conv_step(*args)
    assert torch.equal(y, want)
    with pytest.raises(RuntimeError, match="causal_conv_step is not differentiable"):
        y.sum().backward()


@pytest.mark.parametrize("which", [0, 1, 2, 3, 4, 5])
def test_scan_step_has_values_but_no_gradient(which):
    from paper_2607_18020_b200 import sequence as Q
    args = scan_step_args()
    want = Q.selective_scan_step(args[0].clone(), *args[1:])
    args[which].requires_grad_(True)
    y = Q.selective_scan_step(*args)
    assert torch.equal(y, want)
    with pytest.raises(RuntimeError, match="selective_scan_step is not differentiable"):
        y.sum().backward()


def test_steps_without_grad_mode_carry_no_graph():
    from paper_2607_18020_b200 import sequence as Q
    x, window, w, b = conv_step_args()
    state, u, delta, A, B, C = scan_step_args()
    w, A = torch.nn.Parameter(w), torch.nn.Parameter(A)
    with torch.no_grad():
        assert not Q.causal_conv_step(x, window, w, b).requires_grad
        assert not Q.selective_scan_step(state, u, delta, A, B, C).requires_grad
