"""Infinities in the scan where lanes hold more states, or blocks more channels, than there are: what does not exist
must not turn an infinite result into NaN, and must not reach anything else."""
import pytest

torch = pytest.importorskip("torch")
from forms_util import SCAN_TWO
from seq_util import check, d64, scan_ref

pytestmark = pytest.mark.gpu
INF = float("inf")
# states: full lanes (8, 16, 32, 64) and every kind of padding; 5 and 70 channels fill no block, 128 do
STATES = [1, 3, 4, 5, 8, 12, 16, 24, 33, 64]


def positive(*s, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.rand(*s, generator=g, device="cuda") + 0.1


def inputs(batch, length, channels, n, dtype, seed=31):
    u, delta, z, go = (positive(batch, length, channels, seed=seed + k).to(dtype) for k in range(4))
    B, C = (positive(batch, length, n, seed=seed + 4 + k).to(dtype) for k in range(2))
    return u, delta, -positive(channels, n, seed=seed + 6), B, C, z, go, positive(batch, channels, n, seed=seed + 7)


def run(t, go=None):
    from paper_2607_18020_b200 import sequence as Q
    u, delta, A, B, C, z, _, s = t
    out, last, kept = Q.selective_scan_fwd(u, delta, A, B, C, z=z, state=s, keep=True)
    g = Q.selective_scan_bwd(t[6] if go is None else go, u, delta, A, B, C, z=z, state=s, kept=kept)
    return out, last, g


def split(got, clean, hit):
    """Infinite where `hit`, what it was everywhere else."""
    assert bool((got[hit] == INF).all()), got[hit]
    assert torch.equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("channels", [5, 70, 128])
@pytest.mark.parametrize("n", STATES)
def test_infinite_input(n, channels, dtype):
    """u[1, 20, 3] = inf: that channel's state and output are infinite from there on."""
    t = inputs(2, 41, channels, n, dtype)
    out, last, g = run(t)
    t[0][1, 20, 3] = INF
    out2, last2, g2 = run(t)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[1, 20:, 3] = True
    split(out2, out, hit)
    split(g2.z, g.z, hit)             # without D: D u is no term of the result then, nor 0 times infinity
    rows = torch.zeros_like(last, dtype=torch.bool)
    rows[1, 3] = True
    split(last2, last, rows)
    # gC = sum over channels of h gy: infinite from that node on.  gu and gB see u only at the node itself
    nodes = torch.zeros_like(g.C, dtype=torch.bool)
    nodes[1, 20:] = True
    split(g2.C, g.C, nodes)
    nodes[:] = False
    nodes[1, 20] = True
    split(g2.B, g.B, nodes)
    assert torch.equal(g2.u, g.u)


@pytest.mark.parametrize("size", SCAN_TWO)
def test_infinite_input_where_threads_have_two_channels(size):
    batch, length, channels, n = size
    t = inputs(batch, length, channels, n, torch.float32)
    out, last, g = run(t)
    t[0][batch - 1, 10, channels - 1] = INF
    out2, last2, g2 = run(t)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[-1, 10:, -1] = True
    split(out2, out, hit)
    split(g2.z, g.z, hit)
    rows = torch.zeros_like(last, dtype=torch.bool)
    rows[-1, -1] = True
    split(last2, last, rows)
    nodes = torch.zeros_like(g.C, dtype=torch.bool)
    nodes[-1, 10:] = True
    split(g2.C, g.C, nodes)
    assert torch.equal(g2.u, g.u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("channels", [5, 70, 128])
@pytest.mark.parametrize("n", STATES)
def test_infinite_gradient(n, channels, dtype):
    """gout[0, 20, 1] = inf: the adjoint state of that channel is infinite at that node and before it."""
    t = inputs(2, 41, channels, n, dtype, seed=41)
    _, _, g = run(t)
    go = t[6].clone()
    go[0, 20, 1] = INF
    _, _, g2 = run(t, go)
    hit = torch.zeros_like(g.u, dtype=torch.bool)
    hit[0, :21, 1] = True
    split(g2.u, g.u, hit)
    nodes = torch.zeros_like(g.B, dtype=torch.bool)
    nodes[0, :21] = True
    split(g2.B, g.B, nodes)
    nodes[:] = False
    nodes[0, 20] = True
    split(g2.C, g.C, nodes)
    rows = torch.zeros_like(g.state, dtype=torch.bool)
    rows[0, 1] = True
    split(g2.state, g.state, rows)


@pytest.mark.parametrize("n", STATES)
def test_infinite_projections(n):
    """B[0, 20, n-1] = inf, or C: that state of every channel."""
    t = inputs(1, 41, 128, n, torch.float32, seed=51)
    _, _, g = run(t)
    keep = t[3].clone()
    t[3][0, 20, n - 1] = INF
    out, last, g2 = run(t)
    assert bool((out[0, 20:] == INF).all()) and bool(torch.isfinite(out[0, :20]).all()) and bool((last[..., n - 1] == INF).all())
    hit = torch.zeros_like(g.C, dtype=torch.bool)
    hit[0, 20:, n - 1] = True
    split(g2.C, g.C, hit)
    assert torch.equal(g2.B, g.B)
    t = t[:3] + (keep,) + t[4:]
    t[4][0, 20, n - 1] = INF
    _, _, g2 = run(t)
    hit = torch.zeros_like(g.B, dtype=torch.bool)
    hit[0, :21, n - 1] = True
    split(g2.B, g.B, hit)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", STATES)
def test_infinite_input_of_one_node(n, dtype):
    from paper_2607_18020_b200 import sequence as Q
    u, delta, A, B, C, z, _, s = inputs(2, 1, 70, n, dtype, seed=61)
    a, b = s.clone(), s.clone()
    clean = Q.selective_scan_step(a, u[:, 0], delta[:, 0], A, B[:, 0], C[:, 0], z=z[:, 0])
    u[1, 0, 3] = INF
    out = Q.selective_scan_step(b, u[:, 0], delta[:, 0], A, B[:, 0], C[:, 0], z=z[:, 0])
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[1, 3] = True
    split(out, clean, hit)
    rows = torch.zeros_like(s, dtype=torch.bool)
    rows[1, 3] = True
    split(b, a, rows)


@pytest.mark.parametrize("n", STATES)
def test_infinite_step(n):
    """delta = inf: exp(dt A) is 0 and dt u B infinite, whatever the state was."""
    t = inputs(1, 41, 5, n, torch.float32, seed=71)
    out, last, _ = run(t)
    t[1][0, 20, 2] = INF
    out2, last2, _ = run(t)
    want, wlast = scan_ref(d64(t[0]), d64(t[1]), d64(t[2]), d64(t[3]), d64(t[4]), None, d64(t[5]), None, True, d64(t[7]))
    hit = torch.isinf(want).cuda()
    assert bool(hit[0, 20:, 2].all()) and int(hit.sum()) == 21
    split(out2, out, hit)
    assert bool((last2[0, 2] == INF).all())
    check("the others", out2[~hit], want[~hit.cpu()])
