"""A wait inside linear attention's products that nothing ends: its block gives up, lets what it has issued end, and says so in its
results; the next call is right."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
from attention_forms import ONE, PIECES, linear_forms

pytestmark = pytest.mark.gpu


def call(case, ends, with_state):
    """(o, last state) of fpde_diag_linear_lost, or of the ordinary call where `ends` is None."""
    from paper_2607_18020_b200 import binding as B
    batch, length, heads, dk, dv = case
    g = torch.Generator(device="cuda")
    g.manual_seed(91)
    pad = [-n % 8 for n in (dk, dv)]
    q, k = (torch.randn(batch, length, heads, dk + pad[0], generator=g, device="cuda").bfloat16()[..., :dk] for _ in range(2))
    v = torch.randn(batch, length, heads, dv + pad[1], generator=g, device="cuda").bfloat16()[..., :dv]
    ld = torch.full((heads,), -0.01, device="cuda")
    o = torch.zeros(batch, length, heads, dv, dtype=torch.bfloat16, device="cuda")
    last = torch.zeros(batch, heads, dk, dv, device="cuda") if with_state else None
    a = B.LinearArgs(dtype=B.DTYPE_IDS["torch.bfloat16"], batch=batch, length=length, heads=heads, dk=dk, dv=dv, scale=0.1)
    for name, t in (("q", q), ("k", k), ("v", v)):
        setattr(a, name, t.data_ptr())
        for axis, stride in zip(("batch", "node", "head"), t.stride()):
            setattr(a, "%s_%s" % (name, axis), stride)
    a.log_decay, a.o, a.state_out = ld.data_ptr(), o.data_ptr(), None if last is None else last.data_ptr()
    ws = torch.empty(max(16, B.lib().fpde_linear_attention_workspace_bytes(ctypes.byref(a), 0)), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    stream = torch.cuda.current_stream().cuda_stream
    if ends is None:
        assert B.lib().fpde_linear_attention_fwd(ctypes.byref(a), stream) == 0
    else:
        assert B.lib().fpde_diag_linear_lost(ctypes.byref(a), int(ends), stream) == 0
    torch.cuda.synchronize()
    return o, last


@pytest.mark.parametrize("with_state", [True, False])
@pytest.mark.parametrize("case", ONE + PIECES[:1] + PIECES[2:3] + PIECES[4:5] + PIECES[6:7])
def test_a_march_that_loses_a_wait(case, with_state):
    from paper_2607_18020_b200 import binding as B
    clean, end = call(case, None, with_state)
    before = B.diag_linear_timeouts()
    o, last = call(case, False, with_state)
    pieces, mma = linear_forms("bfloat16", *case)[0]
    assert mma and B.diag_linear_timeouts() == before + case[0] * case[2] * pieces
    assert bool(torch.isnan(o).all()) and (last is None or bool(torch.isnan(last).all()))
    again, end2 = call(case, None, with_state)
    assert torch.equal(again, clean) and bool(torch.isfinite(again).all()) and (end is None or torch.equal(end, end2))
    assert B.diag_linear_timeouts() == before + case[0] * case[2] * pieces


@pytest.mark.parametrize("with_state", [True, False])
@pytest.mark.parametrize("case", PIECES)
def test_ends_that_lose_a_wait(case, with_state):
    """Each row's first piece starts from no end; the others, and the last state, have none to start from."""
    from paper_2607_18020_b200 import binding as B
    batch, length, heads, dk, dv = case
    clean, end = call(case, None, with_state)
    before = B.diag_linear_timeouts()
    o, last = call(case, True, with_state)
    pieces = linear_forms("bfloat16", *case)[0][0]
    assert pieces > 1 and B.diag_linear_timeouts() == before + batch * heads * (pieces - 1)
    first = -(-(-(-length // 128)) // pieces) * 128                  # whole chunks of 128 nodes, as even as they go
    assert torch.equal(o[:, :first], clean[:, :first]) and bool(torch.isnan(o[:, first:]).all())
    assert last is None or bool(torch.isnan(last).all())
    again, end2 = call(case, None, with_state)
    assert torch.equal(again, clean) and (end is None or torch.equal(end, end2))


def test_nothing_is_lost_where_there_is_no_such_wait():
    """Rows in one piece have no ends, and rows of few nodes take 32-bit arithmetic."""
    from paper_2607_18020_b200 import binding as B
    before = B.diag_linear_timeouts()
    for case, ends in ((ONE[0], True), ((1, 9, 2, 16, 16), False), ((1, 9, 2, 16, 16), True)):
        for a, b in zip(call(case, None, True), call(case, ends, True)):
            assert torch.equal(a, b)
    assert B.diag_linear_timeouts() == before
