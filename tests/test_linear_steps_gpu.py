"""Linear attention node by node over thousands of nodes: a step's decay is as exact as the chunked march's."""
import pytest

torch = pytest.importorskip("torch")
from seq_util import FP32, rel

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


@pytest.mark.parametrize("dtype,dk,dv", [(torch.float32, 64, 64), (torch.bfloat16, 48, 33)])
def test_thousands_of_steps_lose_no_digits(dtype, dk, dv):
    """A head that hardly forgets, marched node by node.  A step rounds the state twice, by 2^-24 of itself at most and to either side:
    2^-24 sqrt(2 N) = 1e-5 at most after N = 12345 of them, in the mean a third of it, as roundings are smaller than their largest
    and the state grows with sqrt(N).  One rounding of g to 32 bits, the same in every step, would be 2^-25 N / 2 = 2e-4."""
    from paper_2607_18020_b200 import sequence as Q
    r = gen(61)
    length = 12345
    q, k, v = (r(1, length, 3, n).to(dtype) for n in (dk, dk, dv))
    ld = torch.tensor([-1e-5, -3e-4, -1e-4], device="cuda")
    state = torch.zeros(1, 3, dk, dv, device="cuda")
    for t in range(length):
        o = Q.linear_attention_step(state, q[:, t], k[:, t], v[:, t], ld, 0.125)
    w = torch.exp(ld.double()[:, None] * torch.arange(length - 1, -1, -1, device="cuda"))
    want = torch.einsum("hl,blhi,blhj->bhij", w, k.double(), v.double())
    for h in range(3):
        assert rel(state[:, h], want[:, h]) <= FP32
    assert rel(Q.linear_attention_fwd(q, k, v, ld, 0.125)[1], state) <= FP32
    last = 0.125 * torch.einsum("bhi,bhij->bhj", q[:, -1].double(), want)
    assert rel(o, last) <= 1e-4 if dtype == torch.float32 else rel(o, last) <= 2.0 ** -8 + 1e-4


def test_a_decay_past_the_range_of_32_bits():
    """g is infinite in 32 bits, a state that is not zero with it; one of zeros is 0 times infinity, as the formula has it."""
    from paper_2607_18020_b200 import sequence as Q
    one = torch.ones(1, 1, 4, device="cuda")
    state = torch.ones(1, 1, 4, 4, device="cuda")
    Q.linear_attention_step(state, one, one, one, torch.tensor([100.0], device="cuda"))
    assert bool(torch.isposinf(state).all())
    state = torch.full((1, 1, 4, 4), 3.0, device="cuda")
    Q.linear_attention_step(state, one, one, one, torch.tensor([-float("inf")], device="cuda"))
    assert torch.equal(state, torch.ones_like(state))
