"""Long sums of the fp32 orthogonalisation, and the bits of the 16-bit types' factors.

Sums.  A tensor core cuts the running sum off at every 16-deep product, always towards zero.  Rows that are equal and positive
show it undiluted: X X^T has the one singular value 1, every partial sum is positive, and after ONE step
X1 = (a + b + c) X, so a relative error e of X X^T moves X1 by |b + 2c| / |a + b + c| e = 1.02 e.

Bound, with sums that leave their accumulator every 1024 of depth and at most 64 rows, each term at its worst:
64 products of a segment, cut off by at most 2^-23 of a partial sum that is half the whole on average, 3.9e-6; at most 69
segments added in fp32, 2.1e-6; 22-bit factors of X, 0.24e-6, and of P (2.74 / 0.70 times), 0.93e-6; the four products
of S S and of P X, 0.7e-6 and 0.93e-6; the added term a X, 0.3e-6.  Together 9.1e-6, inside the 1e-5 that every fp32 result is
held to.  One accumulator for all 4376 products of 70001 columns would be off by 1.3e-4 on average.

Bits.  The iteration is carried out in 64 bits with its factors rounded to the bits that fpde.h states, and the kernels'
error may be a tenth larger than that one's: both are rounding errors of the same number of bits in the same places, over
thousands of elements (a spread of a few percent), and fp32 sums add 1e-5 to 2e-3."""
import pytest

torch = pytest.importorskip("torch")
from seq_util import ortho_ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [(1, 33, 70001), (1, 64, 20000), (8, 48, 9000), (1, 70001, 20), (150, 64, 3000)])
def test_long_sums_leave_their_accumulators(size):
    from paper_2607_18020_b200 import optim
    count, rows, cols = size
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    long = torch.rand(count, max(rows, cols), generator=g, device="cuda") + 0.5
    m = long[:, None, :].expand(size) if cols > rows else long[:, :, None].expand(size)
    x = optim.orthogonalize(m.contiguous(), steps=1, eps=0.0)
    want = ortho_ref(m.double(), 1, 0.0)
    for k in range(count):
        r = float(torch.linalg.vector_norm(x[k].double() - want[k]) / torch.linalg.vector_norm(want[k]))
        assert r <= 1e-5, (k, r)


def rounded(x, bits):
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2.0 ** bits) / 2.0 ** bits, e)


def stated(g):
    """The iteration on a stack of 16-bit matrices with the stated bits, in 64-bit arithmetic."""
    x = g / torch.linalg.vector_norm(g, dim=(1, 2), keepdim=True)
    turned = g.shape[1] > g.shape[2]
    x = x.mT if turned else x
    short, long = x.shape[1:]
    padded, small = (short + 63) // 64 * 64, short <= 128 and long <= 256
    all_pairs = small and short <= 8
    square = padded <= 1024 or small
    p_pair, x_pair = padded <= 128 or small, all_pairs or (padded <= 128 and not small)
    a, b, c = 3.4445, -4.775, 2.0315
    for _ in range(5):
        x22, x11 = rounded(x, 22), rounded(x, 11)
        f = x22 if all_pairs else x11
        s = rounded(f @ f.mT, 22)
        t = s if square else rounded(s, 11)
        p = b * s + c * (t @ t)
        x = a * x22 + rounded(p, 22 if p_pair else 11) @ (x22 if x_pair else x11)
    return x.mT if turned else x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [(2000, 8, 8), (500, 16, 40), (200, 40, 40), (100, 64, 200), (30, 200, 64), (30, 128, 256), (40, 32, 300), (20, 64, 900),
                                  (10, 300, 100), (10, 200, 200), (4, 512, 512), (2, 600, 900), (1, 1000, 1030), (1, 1300, 1200)])
def test_16_bit_factors_carry_the_bits_they_state(size, dtype):
    from paper_2607_18020_b200 import optim
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    m = torch.randn(*size, generator=g, device="cuda").to(dtype)
    want = ortho_ref(m.double(), 5, 0.0)

    def mean_error(x):
        return float((torch.linalg.vector_norm(x.double() - want, dim=(1, 2)) / torch.linalg.vector_norm(want, dim=(1, 2))).mean())
    ours, theirs = mean_error(optim.orthogonalize(m, eps=0.0)), mean_error(stated(m.double()).to(dtype))
    assert ours <= 1.1 * theirs + 1e-5, (ours, theirs)
