"""Sizes at which the sequence operators and the orthogonalised update take each form of their kernels, and the questions
to the library which form a call takes, so that no later change of a rule empties the tests of a form."""
import ctypes

from paper_2607_18020_b200 import binding as B

# batch, length, channels, states: two channels a thread in the march, forwards and backwards.  Every number of lanes a
# channel (up to 8, 16, 32, 64 states), full and in part; odd channels; the last two are cut into pieces as well.
SCAN_TWO = [(12, 37, 3201, 5), (12, 37, 3202, 8), (20, 35, 977, 16), (20, 33, 978, 12), (10, 41, 961, 32), (10, 18, 962, 27),
            (6, 35, 801, 64), (6, 20, 802, 40), (1, 700, 1537, 16), (1, 1000, 800, 32)]
# batch, length, channels, width: pieces of more than 16 nodes a thread, and their number
CONV_LONG = [(9, 4097, 2050, 3, 256), (7, 1033, 1351, 4, 32), (7, 1033, 1352, 2, 32), (5, 2100, 2050, 1, 64)]
# batch, channels: four rows a thread in the single-node form, and a last group that is not full
CONV_STEP_ROWS = [(250, 4096), (77, 4095), (1301, 512)]
# count, rows, cols: together every form of every product that 32- and 16-bit matrices take
ORTHO = [(1, 520, 264), (2, 264, 520), (1, 300, 301), (1, 40, 900), (40, 40, 900), (1, 33, 5000), (12, 200, 3000), (1, 1000, 1030),
         (4, 1000, 333), (1, 1500, 700), (24, 300, 300), (1, 2300, 2100), (64, 150, 260), (6, 640, 1280), (1, 700, 4000), (1, 640, 640),
         (1, 448, 512), (1, 384, 1000), (1, 1100, 1200)]


def scan_forms(batch, length, channels, states, backward):
    a = B.ScanArgs(dtype=0, states=states, batch=batch, length=length, channels=channels)
    return B.lib().fpde_diag_scan_channels(ctypes.byref(a), int(backward)), B.lib().fpde_diag_scan_chunks(ctypes.byref(a), int(backward))


def conv_nodes(batch, length, channels, width, backward):
    a = B.ConvArgs(dtype=0, width=width, batch=batch, length=length, channels=channels)
    return B.lib().fpde_diag_conv_nodes(ctypes.byref(a), int(backward))


def conv_step_rows(batch, channels):
    a = B.ConvArgs(dtype=0, width=4, batch=batch, length=1, channels=channels, x_batch=channels)
    return B.lib().fpde_diag_conv_step_rows(ctypes.byref(a))


def ortho_forms(dtype, count, rows, cols):
    a = B.OrthoArgs(dtype=dtype, steps=5, count=count, rows=rows, cols=cols, eps=1e-7)
    return tuple(B.lib().fpde_diag_ortho_form(ctypes.byref(a), p) for p in range(3))
