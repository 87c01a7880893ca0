"""How the sequence operators behave towards autograd beyond their gradients: tensors that single-node calls move
on in place, results that have no gradient, and what is stored for a backward pass that cannot follow."""
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


def test_nothing_is_stored_where_no_backward_pass_can_follow():
    """A, D and the bias of a network in use are parameters: they ask for gradients in every mode."""
    from paper_2607_18020_b200 import sequence as Q
    batch, length, c, n = 2, 2048, 256, 16
    stored = batch * (length // 8) * c * n * 4
    u, delta, z = randn(batch, length, c), randn(batch, length, c), randn(batch, length, c)
    B, C = randn(batch, length, n), randn(batch, length, n)
    A, D, bias = (torch.nn.Parameter(t) for t in (-torch.rand(c, n, device="cuda"), randn(c), randn(c)))
    for needs, mode in ((False, torch.no_grad()), (False, torch.inference_mode()), (True, torch.enable_grad())):
        with mode:
            Q.selective_scan(u, delta, A, B, C, D=D, z=z, delta_bias=bias)
            torch.cuda.synchronize()
            held = torch.cuda.memory_allocated()
            torch.cuda.reset_peak_memory_stats()
            Q.selective_scan(u, delta, A, B, C, D=D, z=z, delta_bias=bias)
            rose = torch.cuda.max_memory_allocated() - held
        assert (rose >= u.numel() * 4 + stored) == needs, (rose, needs)
    with torch.no_grad():
        out = Q.selective_scan(u, delta, A, B, C, D=D, z=z, delta_bias=bias)
    assert not out.requires_grad and torch.equal(out, Q.selective_scan_fwd(u, delta, A, B, C, D, z, bias)[0])
