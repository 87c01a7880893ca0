"""Linear attention head by head and block by block of a row's nodes, and how large its error is over many nodes."""
import math

import pytest

torch = pytest.importorskip("torch")
from attention_blocks import check_all, wanted
from seq_util import rel

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INF = float("inf")
# heads that never forget among ones that do so slowly, within some ten nodes, at once and from node to node
DECAYS = [(-0.004, -0.2, 0.0), (-1.5, -40.0, -INF), (-0.03, -1e-4, 1e-3)]
# rows in one piece and in several, and of few nodes; at least 32 features, so that a node's result is a sum of many terms
CASES = [(1, 700, 64, 64), (1, 520, 128, 128), (2, 300, 32, 64), (1, 450, 128, 40), (1, 261, 64, 112), (3, 60, 64, 64), (1, 33, 128, 64), (1, 128, 64, 64)]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


@pytest.mark.parametrize("states", [True, False])
@pytest.mark.parametrize("decays", DECAYS)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("case", CASES)
def test_every_head_and_block(case, dtype, decays, states):
    batch, length, dk, dv = case
    r = gen(81)
    q, k, v, go = (r(batch, length, 3, n).to(dtype) for n in (dk, dk, dv, dv))
    s, gs = (r(batch, 3, dk, dv), r(batch, 3, dk, dv)) if states else (None, None)
    check_all(q, k, v, torch.tensor(decays, device="cuda"), dk ** -0.5, s, go, gs)


@pytest.mark.parametrize("dim", [64, 128])
def test_two_roundings_and_no_third(dim):
    """bf16 results on the tensor cores have the rounding of one factor of each product and their own.  A rounding to 8 bits is even
    within a step of 2^-7 at a significand's 1: relative to values whose logarithms are even, 2^-7 / sqrt(12) * sqrt(0.75 / (2 ln 2)) =
    1.66e-3 in the mean.  Two that know nothing of each other: 2.35e-3.  A third, as of b's weights with one part of 8 bits
    instead of two or three, makes 2.8e-3 where most of a sum comes through the state.  Samples are many: 5 % over."""
    from paper_2607_18020_b200 import sequence as Q
    one = 2.0 ** -7 / math.sqrt(12) * math.sqrt(0.75 / (2 * math.log(2)))
    lim = 1.05 * math.sqrt(2) * one
    r = gen(82)
    q, k, v, go = (r(1, 1000, 2, dim).to(BF16) for _ in range(4))
    ld = torch.tensor([0.0, -0.001], device="cuda")
    (o, gq, gk, gv), _ = wanted(q, k, v, ld, 0.125, None, go, None)
    g = Q.linear_attention_bwd(go, q, k, v, ld, 0.125)                     # no state leaves any of its marches
    with torch.no_grad():
        without = Q.linear_attention(q, k, v, ld, 0.125)
    results = {"o": (without, o), "o with states": (Q.linear_attention_fwd(q, k, v, ld, 0.125)[0], o), "gq": (g.q, gq), "gk": (g.k, gk), "gv": (g.v, gv)}
    for name, (x, w) in results.items():
        for h in range(2):
            assert rel(x[:, :, h], w[:, :, h]) <= lim, name
