"""Long sums of the fp32 orthogonalisation.

A tensor core cuts the running sum off at every 16-deep product, always towards zero.  Rows that are equal and positive
show it undiluted: X X^T has the one singular value 1, every partial sum is positive, and after ONE step
X1 = (a + b + c) X, so a relative error e of X X^T moves X1 by |b + 2c| / |a + b + c| e = 1.02 e.

Bound, with sums that leave their accumulator every 1024 of depth and at most 64 rows, each term at its worst:
64 products of a segment, cut off by at most 2^-23 of a partial sum that is half the whole on average, 3.9e-6; at most 69
segments added in fp32, 2.1e-6; 22-bit factors of X, 0.24e-6, and of P (2.74 / 0.70 times), 0.93e-6; the four products
of S S and of P X, 0.7e-6 and 0.93e-6; the added term a X, 0.3e-6.  Together 9.1e-6, inside the 1e-5 that every fp32 result is
held to.  One accumulator for all 4376 products of 70001 columns would be off by 1.3e-4 on average."""
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
