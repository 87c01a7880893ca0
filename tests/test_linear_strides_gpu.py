"""Linear attention of bf16 arrays that the copy engine cannot read: odd widths, nodes that are all the same, odd starts."""
import pytest

torch = pytest.importorskip("torch")
from attention_blocks import check_all
from seq_util import GuardedTorch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


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


LD = (-0.004, -0.2, 0.0)


@pytest.mark.parametrize("states", [True, False])
@pytest.mark.parametrize("case", [(1, 1500, 50, 36), (2, 700, 33, 50), (1, 900, 100, 90), (1, 41, 50, 50), (1, 800, 127, 44)])
def test_dense_rows_of_odd_widths(case, states, guard):
    batch, length, dk, dv = case
    r = gen(95)
    q, k, v, go = (r(batch, length, 3, n).to(BF16) for n in (dk, dk, dv, dv))
    s, gs = (r(batch, 3, dk, dv), r(batch, 3, dk, dv)) if states else (None, None)
    check_all(q, k, v, torch.tensor(LD, device="cuda"), dk ** -0.5, s, go, gs)


@pytest.mark.parametrize("how", ["odd rows", "odd start", "one node"])
@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("case", [(1, 1100, 64, 64), (2, 600, 128, 64)])
def test_one_array_of_the_four(case, which, how, guard):
    """The other marches take the tensor cores, and gk the pieces of gv wherever either runs."""
    batch, length, dk, dv = case
    r = gen(96)
    t = [r(batch, length, 3, n).to(BF16) for n in (dk, dk, dv, dv)]
    n = t[which].shape[3]
    if how == "odd rows":
        t[which] = r(batch, length, 3, n + 1).to(BF16)[..., 1:]
    elif how == "odd start":                     # only the launch can see it
        t[which] = r(batch, length, 3, n + 8).to(BF16)[..., 1:n + 1]
    else:
        t[which] = r(batch, 1, 3, n).to(BF16).expand(batch, length, 3, n)
    check_all(*t[:3], torch.tensor(LD, device="cuda"), dk ** -0.5, r(batch, 3, dk, dv), t[3], r(batch, 3, dk, dv))


def test_gradients_of_a_mean_over_the_nodes():
    """Through autograd: what comes back for o has a node stride of zero."""
    from paper_2607_18020_b200 import sequence as Q
    from attention_util import check_attention, linear_ref
    from seq_util import d64
    r = gen(97)
    q, k, v = (r(1, 700, 2, 64).to(BF16).requires_grad_(True) for _ in range(3))
    ld = torch.tensor([-0.01, -0.3], device="cuda")
    up = r(1, 2, 64).to(BF16)
    got = torch.autograd.grad(Q.linear_attention(q, k, v, ld, 0.125).sum(1), (q, k, v), up)
    ref = [d64(t).requires_grad_(True) for t in (q, k, v)]
    want = torch.autograd.grad(linear_ref(*ref, d64(ld), 0.125, None)[0].sum(1), ref, d64(up))
    for name, a, e in zip(("gq", "gk", "gv"), got, want):
        check_attention(name, a, e)
