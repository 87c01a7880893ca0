"""Rows that the copy engine cannot step through are cut for the arithmetic that takes them."""
import ctypes

import pytest

from attention_forms import TYPE, linear_forms
from paper_2607_18020_b200 import binding as B

WIDTH = {"q": "dk", "k": "dk", "v": "dv", "go": "dv"}


def args(dtype, batch, length, heads, dk, dv, **strides):
    """Dense arrays but for those given as (batch, node, head)."""
    a = B.LinearArgs(dtype=TYPE[dtype], batch=batch, length=length, heads=heads, dk=dk, dv=dv, scale=1.0)
    for name, width in WIDTH.items():
        n = getattr(a, width)
        for axis, stride in zip(("batch", "node", "head"), strides.get(name, (length * heads * n, heads * n, n))):
            setattr(a, "%s_%s" % (name, axis), stride)
    return a


def forms(*case, **strides):
    a = args(*case, **strides)
    return [B.lib().fpde_diag_linear_form(ctypes.byref(a), m) for m in range(3)]


@pytest.mark.parametrize("case", [(1, 16384, 16, 50, 50), (1, 4096, 1, 36, 36), (8, 2048, 4, 30, 50), (2, 700, 3, 100, 17), (1, 900, 1, 127, 128)])
def test_dense_rows_of_odd_widths_are_cut_as_those_of_fp16(case):
    assert forms("bfloat16", *case) == forms("float16", *case) and all(n > 0 for n in forms("bfloat16", *case))
    for backward in (0, 1):
        need = [B.lib().fpde_linear_attention_workspace_bytes(ctypes.byref(args(t, *case)), backward) for t in ("bfloat16", "float16")]
        assert need[0] == need[1]


def test_dense_rows_of_whole_16_bytes_are_not():
    case = (1, 16384, 16, 48, 56)
    assert forms("bfloat16", *case) == [-n if mma else n for n, mma in linear_forms("bfloat16", *case)]
    assert all(n < 0 for n in forms("bfloat16", *case))


def test_each_march_by_its_own_arrays():
    """o reads q, k and v; gq go, v and k; gv k, q and go, and gk, in the same pieces, v, go and q."""
    case = (1, 8192, 4, 64, 64)
    plain = forms("float16", *case)
    odd = (8192 * 4 * 65, 4 * 65, 65)
    for name, marches in (("q", (0, 2)), ("k", (0, 1, 2)), ("v", (0, 1, 2)), ("go", (1, 2))):
        got = forms("bfloat16", *case, **{name: odd})
        assert [n > 0 for n in got] == [m in marches for m in range(3)], name
        for m in (0, 1):
            assert got[m] == (plain[m] if m in marches else forms("bfloat16", *case)[m])
        # whole chunks of the tensor cores where one of the two marches is theirs: q and go are read by both
        assert got[2] == plain[2] if name in ("q", "go") else 1 < got[2] <= 8192 // 128


@pytest.mark.parametrize("name,marches", [("go", (1, 2)), ("v", (0, 1, 2))])
def test_all_nodes_the_same(name, marches):
    """What a sum over the nodes hands back, say: its node stride is zero."""
    got = forms("bfloat16", 1, 8192, 4, 64, 64, **{name: (256, 0, 64)})
    assert [n > 0 for n in got] == [m in marches for m in range(3)]
    # but one head for all, or one row, is as good as any
    assert forms("bfloat16", 1, 8192, 4, 64, 64, **{name: (8192 * 64, 64, 0)}) == forms("bfloat16", 1, 8192, 4, 64, 64)


@pytest.mark.parametrize("case", [(1, 16384, 16, 64, 64), (4, 4096, 16, 128, 128)])
def test_the_workspace_is_enough_wherever_the_arrays_start(case):
    """Only the launch sees that an array starts on no multiple of 16 bytes; its march is then cut as fp16's."""
    for backward in (0, 1):
        aligned, odd, fp16 = args("bfloat16", *case), args("bfloat16", *case), args("float16", *case)
        for name in WIDTH:
            setattr(odd, name, 66)
        need = [B.lib().fpde_linear_attention_workspace_bytes(ctypes.byref(a), backward) for a in (aligned, odd, fp16)]
        assert need[0] == need[1] >= need[2] > 0
