"""Rows cut into chunks whose decays leave the range of fp32 while those of their nodes do not: the joined row has to be
what a march through all nodes gives."""
import math

import pytest

torch = pytest.importorskip("torch")
from seq_util import rel

pytestmark = pytest.mark.gpu
LENGTH, CHANNELS, STATES = 4096, 8, 16


def row(step, a, state, go=None, gstate=None, u=0.0):
    """out, last state, gradients of one row with dt = step(t), A = a, B = C = 1."""
    from paper_2607_18020_b200 import sequence as Q
    u = torch.full((1, LENGTH, CHANNELS), u, device="cuda")
    delta = step.reshape(1, LENGTH, 1).expand(1, LENGTH, CHANNELS).contiguous().cuda()
    A = torch.full((CHANNELS, STATES), a, device="cuda")
    B = torch.ones(1, LENGTH, STATES, device="cuda")
    out, last, kept = Q.selective_scan_fwd(u, delta, A, B, B, delta_softplus=False, state=state, keep=True)
    go = torch.zeros_like(u) if go is None else go
    return out, last, Q.selective_scan_bwd(go, u, delta, A, B, B, delta_softplus=False, state=state, kept=kept, gstate=gstate)


def test_these_rows_are_cut():
    import ctypes
    from paper_2607_18020_b200 import binding
    a = binding.ScanArgs(dtype=0, states=STATES, batch=1, length=LENGTH, channels=CHANNELS)
    assert binding.lib().fpde_selective_scan_workspace_bytes(ctypes.byref(a), 0) > 0
    # a chunk is at least 32 nodes long: exp(3 * 32) is past 3.4e38
    assert math.exp(3 * 32) > torch.finfo(torch.float32).max


def test_nothing_grows_from_nothing():
    """A > 0, and neither input nor state: 0 at every node, forwards and backwards."""
    out, last, g = row(torch.full((LENGTH,), 3.0), 1.0, None)
    for t in (out, last, g.u, g.delta, g.A, g.B, g.C):
        assert bool((t == 0).all())


def test_a_state_that_grows_past_a_chunk():
    """exp(96) over the first 32 nodes, nothing after: 1e-35 becomes 4.9e6.  The exponent, 138.5 in powers of two, carries
    two roundings of 2^-24 (log2 e in A, its product with the sum of dt), ln 2 * 138.5 * 2^-23 = 1.15e-5 of the result;
    what every fp32 result is held to, 1e-5, comes on top."""
    step = torch.zeros(LENGTH)
    step[:32] = 3.0
    state = torch.full((1, CHANNELS, STATES), 1e-35, device="cuda")
    want = state.double() * math.exp(96)
    out, last, _ = row(step, 1.0, state)
    assert rel(last, want) <= 2.2e-5
    assert rel(out[:, 32:], (want.sum(-1))[:, None].expand(-1, LENGTH - 32, -1)) <= 2.2e-5
    # the same backwards, from the last nodes
    _, _, g = row(step.flip(0), 1.0, torch.zeros_like(state), gstate=state)
    assert rel(g.state, want) <= 2.2e-5


def test_an_infinite_state_stays():
    """exp(-3) a node: no node's decay is 0, a chunk's is."""
    state = torch.zeros(1, CHANNELS, STATES, device="cuda")
    state[0, 2, 5] = float("inf")
    out, last, g = row(torch.full((LENGTH,), 3.0), -1.0, state, gstate=state)
    for t in (last, g.state):
        assert bool((t[0, 2, 5] == float("inf"))) and int(torch.isinf(t).sum()) == 1 and not bool(torch.isnan(t).any())
    assert bool((out[0, :, 2] == float("inf")).all()) and int(torch.isinf(out).sum()) == LENGTH and not bool(torch.isnan(out).any())


def test_a_state_that_fades_leaves_what_came_after_it():
    """A finite state is forgotten within a chunk: the steady value of u = 1 is left, as from any other state."""
    a, _, _ = row(torch.full((LENGTH,), 3.0), -1.0, torch.full((1, CHANNELS, STATES), 1e30, device="cuda"), u=1.0)
    steady = STATES * 3.0 / (1 - math.exp(-3.0))
    assert rel(a[:, 128:], torch.full_like(a[:, 128:], steady)) <= 1e-5
