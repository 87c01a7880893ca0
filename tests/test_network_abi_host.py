"""Sequence operators and orthogonalised updates without a GPU: layout of the argument blocks, size
queries, refusals with the documented status codes, and the Python layer's own checks."""
import ctypes
import os
import subprocess

import pytest

from paper_2607_18020_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, ALIGN, WORKSPACE, DTYPE, PARAM = 2, 4, 5, 9, 11, 12


def test_argument_blocks_match_the_header(tmp_path):
    names = {"fpde_conv_args": B.ConvArgs, "fpde_scan_args": B.ScanArgs, "fpde_ortho_args": B.OrthoArgs}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "fpde.h"', "int main(void) {"]
    for c, py in names.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (c, c))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (c, f[0], c, f[0]) for f in py._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    exe = str(tmp_path / "layout")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", exe, str(src)])
    said = dict(line.split() for line in subprocess.check_output([exe], text=True).splitlines())
    for c, py in names.items():
        assert int(said[c]) == ctypes.sizeof(py)
        for f in py._fields_:
            assert int(said["%s.%s" % (c, f[0])]) == getattr(py, f[0]).offset, f[0]


def conv(**k):
    base = dict(dtype=0, width=4, silu=1, batch=2, length=9, channels=6, x=64, x_batch=54, x_node=6, weight=64, state=64, y=64, state_out=128,
                gy=64, gy_batch=54, gy_node=6, gx=64, gweight=64)
    return B.ConvArgs(**{**base, **k})


def scan(**k):
    base = dict(dtype=0, states=16, softplus=1, batch=2, length=40, channels=6, A=64, out=64, gout=64, gu=64, gdelta=64, gB=64, gC=64, gA=64)
    for n in ("u", "delta", "B", "C"):
        base[n] = 64
    return B.ScanArgs(**{**base, **k})


def ortho(**k):
    return B.OrthoArgs(**{**dict(dtype=0, steps=5, count=1, rows=300, cols=300, grad=64, grad_matrix=90000, grad_row=300, out=64, weight=64,
                                 momentum=64, eps=1e-7, lr=0.1), **k})


def status(name, args):
    return getattr(B.lib(), name)(ctypes.byref(args) if args is not None else None, None)


@pytest.mark.parametrize("name,make", [("fpde_causal_conv_fwd", conv), ("fpde_causal_conv_bwd", conv), ("fpde_causal_conv_step", conv),
                                       ("fpde_selective_scan_fwd", scan), ("fpde_selective_scan_bwd", scan), ("fpde_selective_scan_step", scan),
                                       ("fpde_orthogonalize", ortho), ("fpde_muon_step", ortho)])
def test_common_refusals(name, make):
    assert status(name, None) == NULL
    assert status(name, make(dtype=3)) == DTYPE
    assert status(name, make(dtype=-1)) == DTYPE
    big = {"count": -1} if make is ortho else {"batch": -1}
    assert status(name, make(**big)) == SHAPE


def test_conv_refusals():
    assert status("fpde_causal_conv_fwd", conv(width=0)) == PARAM
    assert status("fpde_causal_conv_fwd", conv(width=5)) == PARAM
    assert status("fpde_causal_conv_fwd", conv(x=None)) == NULL
    assert status("fpde_causal_conv_fwd", conv(y=None)) == NULL
    assert status("fpde_causal_conv_fwd", conv(x=66)) == ALIGN
    assert status("fpde_causal_conv_fwd", conv(state_out=64)) == PARAM      # the window is read by other blocks
    assert status("fpde_causal_conv_bwd", conv(gweight=None)) == NULL
    assert status("fpde_causal_conv_bwd", conv()) == WORKSPACE
    assert status("fpde_causal_conv_step", conv(weight=None)) == NULL


def test_scan_refusals():
    assert status("fpde_selective_scan_fwd", scan(states=0)) == PARAM
    assert status("fpde_selective_scan_fwd", scan(states=65)) == PARAM
    assert status("fpde_selective_scan_fwd", scan(A=None)) == NULL
    assert status("fpde_selective_scan_fwd", scan(out=None)) == NULL
    assert status("fpde_selective_scan_fwd", scan(u=65)) == ALIGN
    assert status("fpde_selective_scan_fwd", scan(kept=72, kept_bytes=1 << 20)) == WORKSPACE
    assert status("fpde_selective_scan_fwd", scan(kept=64, kept_bytes=8)) == WORKSPACE
    assert status("fpde_selective_scan_bwd", scan()) == WORKSPACE                    # no stored states
    assert status("fpde_selective_scan_bwd", scan(kept=64, kept_bytes=1 << 20)) == WORKSPACE
    assert status("fpde_selective_scan_bwd", scan(kept=64, kept_bytes=1 << 20, z=64)) == NULL
    assert status("fpde_selective_scan_step", scan(B=None)) == NULL


def test_ortho_refusals():
    assert status("fpde_orthogonalize", ortho(steps=-1)) == PARAM
    assert status("fpde_orthogonalize", ortho(steps=101)) == PARAM
    assert status("fpde_orthogonalize", ortho(eps=float("nan"))) == PARAM
    assert status("fpde_orthogonalize", ortho(grad=None)) == NULL
    assert status("fpde_orthogonalize", ortho()) == WORKSPACE
    assert status("fpde_orthogonalize", ortho(out=66)) == ALIGN
    assert status("fpde_muon_step", ortho(momentum=None)) == NULL
    assert status("fpde_muon_step", ortho(workspace=128, workspace_bytes=1 << 30)) == WORKSPACE      # 256-byte aligned


def test_nothing_to_do_is_no_error_and_needs_no_device():
    assert status("fpde_causal_conv_fwd", conv(batch=0)) == 0
    assert status("fpde_causal_conv_step", conv(channels=0)) == 0
    assert status("fpde_selective_scan_fwd", scan(channels=0)) == 0
    assert status("fpde_orthogonalize", ortho(rows=0)) == 0


def test_size_queries():
    L = B.lib()
    per = 6 * 16 * 4
    assert L.fpde_selective_scan_kept_bytes(ctypes.byref(scan(length=0))) == 0
    assert L.fpde_selective_scan_kept_bytes(ctypes.byref(scan(length=1))) == 2 * per
    assert L.fpde_selective_scan_kept_bytes(ctypes.byref(scan(length=17))) == 2 * 3 * per
    assert L.fpde_selective_scan_workspace_bytes(ctypes.byref(scan()), 0) == 0          # a short row is not split
    assert L.fpde_selective_scan_workspace_bytes(ctypes.byref(scan(length=100000)), 0) > 0
    assert L.fpde_selective_scan_workspace_bytes(ctypes.byref(scan()), 1) > 0
    assert L.fpde_causal_conv_workspace_bytes(ctypes.byref(conv())) == 2 * 6 * 5 * 4
    assert L.fpde_causal_conv_workspace_bytes(ctypes.byref(conv(width=9))) == 0
    assert L.fpde_orthogonalize_workspace_bytes(ctypes.byref(ortho(rows=128, cols=256))) == 0       # stays on one SM
    assert L.fpde_orthogonalize_workspace_bytes(ctypes.byref(ortho(rows=129, cols=129))) > 0
    # offsets past 32 bits: sizes of long rows are formed in 64
    assert L.fpde_selective_scan_kept_bytes(ctypes.byref(scan(length=1 << 34))) == 2 * (1 << 31) * per


def test_python_layer_refuses_cpu_tensors():
    torch = pytest.importorskip("torch")
    from paper_2607_18020_b200 import optim, sequence
    x, w = torch.ones(2, 5, 6), torch.ones(6, 4)
    with pytest.raises(ValueError):
        sequence.causal_conv_fwd(x, w)
    with pytest.raises(ValueError):
        sequence.selective_scan_fwd(x, x, torch.ones(6, 16), torch.ones(2, 5, 16), torch.ones(2, 5, 16))
    with pytest.raises(ValueError):
        optim.orthogonalize(w)
    with pytest.raises(ValueError):
        optim.Muon([torch.nn.Parameter(torch.ones(3))])
