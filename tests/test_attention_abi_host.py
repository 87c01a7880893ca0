"""Rotation, norm of heads and linear attention without a GPU: layout of the argument blocks, size queries, refusals with the
documented status codes."""
import ctypes
import os
import subprocess

import pytest

from paper_2607_18020_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, ALIGN, WORKSPACE, DTYPE, PARAM = 0, 2, 4, 5, 9, 11, 12


def test_argument_blocks_match_the_header(tmp_path):
    names = {"fpde_head_args": B.HeadArgs, "fpde_linear_args": B.LinearArgs}
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


def head(**k):
    base = dict(dtype=0, norm=1, pairs=4, batch=2, length=9, q_heads=3, k_heads=1, dim=16, eps=1e-6, inv_freq=64)
    base.update({n: 64 for n in ("q", "k", "q_out", "k_out", "gq", "gk", "gx_q", "gx_k", "gq_weight", "gk_weight")})
    return B.HeadArgs(**{**base, **k})


def linear(**k):
    base = dict(dtype=0, batch=2, length=9, heads=3, dk=16, dv=24, scale=1.0, log_decay=64, state=64, state_out=128, gstate_out=64, gstate=128)
    base.update({n: 64 for n in ("q", "k", "v", "o", "go", "gq", "gk", "gv")})
    return B.LinearArgs(**{**base, **k})


def status(name, args):
    return getattr(B.lib(), name)(ctypes.byref(args) if args is not None else None, None)


HEAD = ("fpde_head_rotary_fwd", "fpde_head_rotary_bwd")
LINEAR = ("fpde_linear_attention_fwd", "fpde_linear_attention_bwd", "fpde_linear_attention_step")


@pytest.mark.parametrize("name,make", [(n, head) for n in HEAD] + [(n, linear) for n in LINEAR])
def test_common_refusals(name, make):
    assert status(name, None) == NULL
    assert status(name, make(dtype=3)) == DTYPE
    assert status(name, make(dtype=-1)) == DTYPE
    assert status(name, make(batch=-1)) == SHAPE
    assert status(name, make(length=-1, **({"batch": 1} if make is head else {}))) == SHAPE
    assert status(name, make(batch=(1 << 36) + 1)) == SHAPE
    assert status(name, make(q=66)) == ALIGN if name not in HEAD[1:] else True


@pytest.mark.parametrize("name", HEAD)
def test_head_refusals(name):
    assert status(name, head(dim=0)) == PARAM
    assert status(name, head(dim=257)) == PARAM
    assert status(name, head(pairs=9)) == PARAM
    assert status(name, head(pairs=-1)) == PARAM
    assert status(name, head(eps=-1.0)) == PARAM
    assert status(name, head(eps=float("nan"))) == PARAM
    assert status(name, head(inv_freq=None)) == NULL
    assert status(name, head(positions=68)) == ALIGN
    assert status(name, head(q_weight=66)) == ALIGN
    assert status(name, head(q_heads=-1)) == SHAPE


def test_head_refusals_of_one_direction():
    assert status(HEAD[0], head(q=None)) == NULL
    assert status(HEAD[0], head(k=None)) == NULL
    assert status(HEAD[0], head(k_out=None)) == NULL
    assert status(HEAD[0], head(q_out=66)) == ALIGN
    assert status(HEAD[1], head(gq=None)) == NULL
    assert status(HEAD[1], head(gx_k=None)) == NULL
    assert status(HEAD[1], head(q=None)) == NULL
    assert status(HEAD[1], head()) == WORKSPACE
    need = B.lib().fpde_head_rotary_workspace_bytes(ctypes.byref(head()))
    assert need > 0 and B.lib().fpde_head_rotary_workspace_bytes(ctypes.byref(head(norm=0))) == 0
    assert status(HEAD[1], head(workspace=64, workspace_bytes=need - 1)) == WORKSPACE
    assert status(HEAD[1], head(workspace=72, workspace_bytes=need)) == WORKSPACE
    for empty in (dict(batch=0), dict(length=0), dict(q_heads=0, k_heads=0)):
        assert status(HEAD[0], head(**empty)) == OK          # nothing to launch
        assert status(HEAD[1], head(norm=0, **empty)) == OK


def test_linear_refusals():
    for name in LINEAR:
        assert status(name, linear(dk=0)) == PARAM
        assert status(name, linear(dv=129)) == PARAM
        assert status(name, linear(scale=float("inf"))) == PARAM
        assert status(name, linear(log_decay=None)) == NULL
        assert status(name, linear(v=None)) == NULL
        assert status(name, linear(state=66)) == ALIGN
        assert status(name, linear(batch=0)) == OK
        assert status(name, linear(heads=0)) == OK
    assert status(LINEAR[0], linear(o=None)) == NULL
    assert status(LINEAR[0], linear(state=128)) == PARAM         # blocks still read it
    assert status(LINEAR[1], linear(go=None)) == NULL
    assert status(LINEAR[1], linear(gv=None)) == NULL
    assert status(LINEAR[1], linear(gstate=64)) == PARAM
    assert status(LINEAR[2], linear(o=None)) == NULL


def test_linear_workspace():
    need = lambda backward=0, **k: B.lib().fpde_linear_attention_workspace_bytes(ctypes.byref(linear(**k)), backward)    # noqa: E731
    assert need() == 0                                           # a short row is not cut
    assert need(dk=129) == 0
    long = dict(batch=1, length=20000, heads=2, dk=64, dv=64)
    assert need(**long) > 0 and need(1, **long) > 0
    assert status(LINEAR[0], linear(**long)) == WORKSPACE
    assert status(LINEAR[0], linear(workspace=64, workspace_bytes=need(**long) - 1, **long)) == WORKSPACE
    assert status(LINEAR[1], linear(workspace=72, workspace_bytes=1 << 40, **long)) == WORKSPACE
