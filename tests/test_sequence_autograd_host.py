"""When the scan is asked to store what its backward pass needs, without a GPU: a stand-in takes the kernels' place."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def asked(monkeypatch):
    from paper_2607_18020_b200 import sequence as Q
    seen = []

    def stand_in(u, delta, A, B, C, D=None, z=None, delta_bias=None, delta_softplus=True, state=None, keep=False):
        seen.append(keep)
        return u * 2, torch.zeros(u.shape[0], *A.shape), torch.zeros(1) if keep else None
    monkeypatch.setattr(Q, "selective_scan_fwd", stand_in)
    return seen


def tensors():
    return torch.ones(2, 5, 3), torch.ones(2, 5, 3), -torch.ones(3, 4), torch.ones(2, 5, 4), torch.ones(2, 5, 4)


@pytest.mark.parametrize("which", [0, 1, 2, 3, 4])
def test_states_are_kept_only_where_a_backward_pass_can_follow(asked, which):
    from paper_2607_18020_b200 import sequence as Q
    t = list(tensors())
    Q.selective_scan(*t)
    t[which] = torch.nn.Parameter(t[which])
    assert Q.selective_scan(*t).requires_grad
    for mode in (torch.no_grad(), torch.inference_mode()):
        with mode:
            assert not Q.selective_scan(*t).requires_grad
    assert asked == [False, True, False, False]


def test_a_parameter_among_the_optional_tensors_counts(asked):
    from paper_2607_18020_b200 import sequence as Q
    t = tensors()
    for name, shape in (("D", (3,)), ("z", (2, 5, 3)), ("delta_bias", (3,)), ("state", (2, 3, 4))):
        Q.selective_scan(*t, **{name: torch.nn.Parameter(torch.ones(shape))})
    assert asked == [True] * 4
