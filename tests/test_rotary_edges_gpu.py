"""Rotation by frequencies that are no numbers."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs", [(32, 16), (33, 5), (128, 32)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_frequency_that_is_no_number_makes_its_pair_nan(bad, dim, pairs, interleaved):
    """cos and sin of such an angle are NaN, and so is the pair that they turn, at every node but nowhere else."""
    from paper_2607_18020_b200 import sequence as Q
    g = torch.Generator(device="cuda")
    g.manual_seed(71)
    q, w = torch.randn(2, 70, 3, dim, generator=g, device="cuda"), torch.randn(dim, generator=g, device="cuda")
    freq = Q.rotary_frequencies(pairs)
    broken = freq.clone()
    broken[3] = bad
    mine = [6, 7] if interleaved else [3, 3 + pairs]
    others = [i for i in range(dim) if i not in mine]

    def calls(f):
        yield Q.rotary_fwd(q, None, f, offset=5, interleaved=interleaved)[0]
        yield Q.rotary_bwd(q, None, f, offset=5, interleaved=interleaved)[0]
        yield Q.norm_rotary_fwd(q, None, w, None, f, offset=5, interleaved=interleaved)[0]
    for got, clean in zip(calls(broken), calls(freq)):
        assert bool(torch.isnan(got[..., mine]).all())
        assert torch.equal(got[..., others], clean[..., others])
    # in the norm's gradient a head's features share a sum
    back = Q.norm_rotary_bwd(q, None, q, None, w, None, broken, offset=5, interleaved=interleaved)
    assert bool(torch.isnan(back.q).all()) and bool(torch.isnan(back.q_weight[mine]).all()) and bool(torch.isfinite(back.q_weight[others]).all())
