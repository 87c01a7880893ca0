"""Sizes at which linear attention takes each form of its kernels, and the question to the library which one a call takes, so
that no later change of a rule empties the tests of a form."""
import ctypes

from paper_2607_18020_b200 import binding as B

TYPE = {"float32": 0, "bfloat16": 1, "float16": 2}
# batch, length, heads, dk, dv: rows of several pieces on the tensor cores, with up to 64 and 128 features on either side, lengths
# that end a piece or a chunk early or just begin one; and such rows in one piece
PIECES = [(1, 1000, 1, 64, 64), (1, 1025, 2, 33, 50), (1, 1000, 1, 128, 40), (1, 897, 1, 65, 64), (1, 700, 2, 40, 128), (1, 769, 1, 64, 72),
          (1, 900, 1, 128, 128), (2, 1153, 1, 96, 104)]
ONE = [(2, 300, 2, 64, 64), (1, 385, 1, 128, 16), (1, 300, 2, 16, 128), (1, 65, 3, 80, 112)]
# the same of 32-bit arithmetic: up to 32, 64 and 128 features of a, up to 32, 64 and more of c
PLAIN = [(1, 300, 1, 32, 32), (2, 197, 3, 20, 9), (1, 130, 1, 64, 32), (1, 131, 2, 128, 24), (1, 129, 2, 32, 64), (1, 161, 1, 64, 64), (1, 200, 2, 100, 64),
         (1, 200, 1, 31, 128), (1, 140, 2, 64, 100), (1, 300, 1, 128, 128)]
# in one piece forwards and in several backwards
MIXED = [(2, 97, 3, 20, 9), (1, 100, 2, 100, 64), (1, 100, 1, 31, 128)]


def linear_forms(dtype, batch, length, heads, dk, dv):
    """(pieces of a row, on the tensor cores) of the marches of o, gq, and gv with gk."""
    a = B.LinearArgs(dtype=TYPE[dtype], batch=batch, length=length, heads=heads, dk=dk, dv=dv, scale=1.0)
    n = [B.lib().fpde_diag_linear_form(ctypes.byref(a), m) for m in range(3)]
    return [(abs(x), x < 0) for x in n]
