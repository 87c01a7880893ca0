"""What linear attention and the rotation keep between calls, and the numbers they take, without a GPU: the calls are recorded
instead of queued."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def calls(monkeypatch):
    from paper_2607_18020_b200 import binding, sequence
    queued = []
    monkeypatch.setattr(sequence, "_first", lambda name, t, dims: None)              # CPU tensors stand in
    monkeypatch.setattr(sequence, "_plans", binding.ArgPlans())
    monkeypatch.setattr(binding, "call_with", lambda name, a, device: queued.append(type(a).from_buffer_copy(a)))
    return queued


def attention(Q, scale):
    q, k, v = torch.zeros(1, 9, 2, 16), torch.zeros(1, 9, 2, 16), torch.zeros(1, 9, 2, 8)
    ld, state = torch.zeros(2), torch.zeros(1, 2, 16, 8)
    Q.linear_attention_fwd(q, k, v, ld, scale)
    Q.linear_attention_bwd(v, q, k, v, ld, scale)
    Q.linear_attention_step(state, q[:, 0], k[:, 0], v[:, 0], ld, scale)


def norm(Q, eps):
    q = torch.zeros(1, 9, 2, 16)
    Q.norm_rotary_fwd(q, None, eps=eps)
    Q.norm_rotary_bwd(q, None, q, None, eps=eps)


def rotation(Q, offset):
    q, freq = torch.zeros(1, 9, 2, 16), torch.zeros(8)
    Q.rotary_fwd(q, q, freq, offset=offset)
    Q.rotary_bwd(q, q, freq, offset=offset)
    Q.norm_rotary_fwd(q, q, None, None, freq, offset=offset)
    Q.norm_rotary_bwd(q, q, q, q, None, None, freq, offset=offset)


def test_scale_and_eps_are_those_of_the_call(calls):
    from paper_2607_18020_b200 import sequence as Q
    for x in (0.5, 2, np.float64(0.25), np.float32(0.125), 0.5):
        attention(Q, x)
        norm(Q, x)
        assert [a.scale for a in calls[:3]] == [float(x)] * 3 and [a.eps for a in calls[3:]] == [float(x)] * 2
        calls.clear()


@pytest.mark.parametrize("make", [lambda x: torch.tensor(x), lambda x: np.array(x), lambda x: str(x), lambda x: None])
def test_a_scale_or_eps_that_is_no_number_is_refused(calls, make):
    """A tensor may hold another value in the next call, and could ask for a gradient."""
    from paper_2607_18020_b200 import sequence as Q
    q, k, v, ld, state = torch.zeros(1, 9, 2, 16), torch.zeros(1, 9, 2, 16), torch.zeros(1, 9, 2, 8), torch.zeros(2), torch.zeros(1, 2, 16, 8)
    x = make(0.5)
    for call in (lambda: Q.linear_attention_fwd(q, k, v, ld, x), lambda: Q.linear_attention_bwd(v, q, k, v, ld, x),
                 lambda: Q.linear_attention_step(state, q[:, 0], k[:, 0], v[:, 0], ld, x), lambda: Q.linear_attention(q, k, v, ld, x)):
        with pytest.raises(ValueError, match="scale"):
            call()
    for call in (lambda: Q.norm_rotary_fwd(q, None, eps=x), lambda: Q.norm_rotary_bwd(q, None, q, None, eps=x), lambda: Q.norm_rotary(q, None, eps=x)):
        with pytest.raises(ValueError, match="eps"):
            call()
    assert not calls


def test_the_optimiser_takes_the_eps_of_the_call(monkeypatch):
    """Of a tensor as well, whose value may have changed since a call with the same tensor."""
    from paper_2607_18020_b200 import binding, optim
    queued = []
    monkeypatch.setattr(optim, "_matrices", lambda name, t: t[None] if t.dim() == 2 else t)
    monkeypatch.setattr(binding, "call_with", lambda name, a, device: queued.append(a.eps))
    w, g, m, eps = torch.zeros(8, 4), torch.zeros(8, 4), torch.zeros(8, 4), torch.tensor(0.5)
    for _ in range(2):
        optim.orthogonalize(g, eps=eps)
        optim.muon_step(w, g, m, 0.1, eps=eps)
        eps.mul_(0.5)
    assert queued == [0.5, 0.5, 0.25, 0.25]


def test_a_march_by_offset_keeps_one_plan_a_call(calls):
    """The position of a row that continues is another one in every call, and none of them drives out the plans of other operators."""
    from paper_2607_18020_b200 import sequence as Q
    x, taps = torch.zeros(1, 9, 16), torch.zeros(16, 4)
    Q.causal_conv_fwd(x, taps)
    conv = [k for k in Q._plans._plans]
    assert len(conv) == 1
    for t in range(600):
        rotation(Q, t)
    assert all(k in Q._plans._plans for k in conv) and len(Q._plans._plans) == 5
    assert [a.offset for a in calls[1:]] == [t for t in range(600) for _ in range(4)]


def test_offsets_are_whole_numbers_of_64_bits(calls):
    from paper_2607_18020_b200 import sequence as Q
    ends = (-2 ** 63, -1, 0, np.int64(7), 2 ** 63 - 1)
    for x in ends:
        rotation(Q, x)
    assert [a.offset for a in calls] == [int(x) for x in ends for _ in range(4)]
    calls.clear()
    q, freq = torch.zeros(1, 9, 2, 16), torch.zeros(8)
    for x in (2 ** 63, -2 ** 63 - 1, 2 ** 64, 1.0, "1", None, torch.tensor(3)):
        for call in (lambda: Q.rotary_fwd(q, q, freq, offset=x), lambda: Q.rotary_bwd(q, q, freq, offset=x), lambda: Q.rotary(q, q, freq, offset=x),
                     lambda: Q.norm_rotary_fwd(q, q, None, None, freq, offset=x), lambda: Q.norm_rotary_bwd(q, q, q, q, None, None, freq, offset=x)):
            with pytest.raises(ValueError, match="offset"):
                call()
    assert not calls
