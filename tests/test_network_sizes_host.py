"""Extents whose products pass 64 bits (zero strides let a call have them): refused, not wrapped around."""
import ctypes

import pytest

from paper_2607_18020_b200 import binding as B
from test_network_abi_host import SHAPE, conv, ortho, scan, status


@pytest.mark.parametrize("sizes", [dict(batch=1 << 40, length=1, channels=1 << 24), dict(batch=1 << 40, length=1 << 40, channels=1),
                                   dict(batch=1 << 36, length=1 << 36, channels=1 << 8), dict(batch=1 << 32, length=1 << 8, channels=1 << 9)])
def test_sequence_extents(sizes):
    for name in ("fpde_causal_conv_fwd", "fpde_causal_conv_bwd"):
        assert status(name, conv(**sizes)) == SHAPE, name
    assert B.lib().fpde_causal_conv_workspace_bytes(ctypes.byref(conv(**sizes))) == 0
    for name in ("fpde_selective_scan_fwd", "fpde_selective_scan_bwd"):
        assert status(name, scan(**sizes)) == SHAPE, name
    assert B.lib().fpde_selective_scan_kept_bytes(ctypes.byref(scan(**sizes))) == 0
    for backward in (0, 1):
        assert B.lib().fpde_selective_scan_workspace_bytes(ctypes.byref(scan(**sizes)), backward) == 0


def test_single_nodes():
    """Their length is 1, whatever the argument block says; batch times channels alone is past 2^64, or wraps to 0."""
    assert status("fpde_causal_conv_step", conv(batch=1 << 40, channels=1 << 24)) == SHAPE
    assert status("fpde_selective_scan_step", scan(batch=1 << 36, channels=1 << 24)) == SHAPE


def test_matrix_extents():
    big = dict(count=1 << 20, rows=1 << 20, cols=1 << 20)
    assert status("fpde_orthogonalize", ortho(**big)) == SHAPE and status("fpde_muon_step", ortho(**big)) == SHAPE
    assert B.lib().fpde_orthogonalize_workspace_bytes(ctypes.byref(ortho(**big))) == 0


def test_the_largest_extents_have_sizes():
    """Just inside the limit the sizes are what they are, in 64 bits."""
    n = 1 << 20
    assert B.lib().fpde_selective_scan_kept_bytes(ctypes.byref(scan(batch=n, length=n, channels=256, states=64))) == (n * n // 8) * 256 * 64 * 4
    assert B.lib().fpde_causal_conv_workspace_bytes(ctypes.byref(conv(batch=n, length=n - 4, channels=256))) >= n * 256 * 5 * 4
    assert B.lib().fpde_orthogonalize_workspace_bytes(ctypes.byref(ortho(count=256, rows=n, cols=n))) > 4 * 256 * n * n * 4
