"""The sizes that the GPU tests of linear attention use to reach a form of its kernels still take that form."""
import ctypes

import pytest

from attention_forms import MIXED, ONE, PIECES, PLAIN, linear_forms
from paper_2607_18020_b200 import binding as B


@pytest.mark.parametrize("case", PIECES)
def test_rows_in_pieces_on_tensor_cores(case):
    assert all(mma and pieces > 1 for pieces, mma in linear_forms("bfloat16", *case))


@pytest.mark.parametrize("case", ONE)
def test_rows_in_one_piece_on_tensor_cores(case):
    assert linear_forms("bfloat16", *case)[0] == (1, True)        # of o; a gradient's march may be cut


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("case", PLAIN)
def test_rows_in_pieces_of_32_bit_arithmetic(case, dtype):
    assert all(pieces > 1 and not mma for pieces, mma in linear_forms(dtype, *case))


@pytest.mark.parametrize("case", MIXED)
def test_rows_in_one_piece_forwards_and_several_backwards(case):
    o, *rest = linear_forms("float32", *case)
    assert o == (1, False) and all(pieces > 1 and not mma for pieces, mma in rest)


def test_questions_refused():
    ask = B.lib().fpde_diag_linear_form
    good = dict(dtype=0, batch=1, length=40, heads=1, dk=8, dv=8, scale=1.0)
    assert ask(None, 0) == 0
    assert ask(ctypes.byref(B.LinearArgs(**good)), 3) == 0 and ask(ctypes.byref(B.LinearArgs(**good)), -1) == 0
    assert ask(ctypes.byref(B.LinearArgs(**{**good, "dk": 129})), 0) == 0
    assert ask(ctypes.byref(B.LinearArgs(**good)), 0) > 0
