"""The sizes that the tests of the kernels' forms use do take those forms."""
import pytest

from forms_util import CONV_LONG, CONV_STEP_ROWS, ORTHO, SCAN_TWO, conv_nodes, conv_step_rows, ortho_forms, scan_forms


@pytest.mark.parametrize("size", SCAN_TWO)
def test_two_channels_a_thread(size):
    assert scan_forms(*size, False)[0] == 2 and scan_forms(*size, True)[0] == 2


def test_scans_of_all_kinds_are_among_them():
    lanes = {max(8, 1 << (s[3] - 1).bit_length()) for s in SCAN_TWO}
    assert lanes == {8, 16, 32, 64}
    for n in lanes:
        assert {s[2] % 2 for s in SCAN_TWO if max(8, 1 << (s[3] - 1).bit_length()) == n} == {0, 1}
    assert any(scan_forms(*s, False)[1] > 1 and scan_forms(*s, True)[1] > 1 for s in SCAN_TWO)


@pytest.mark.parametrize("size", CONV_LONG)
def test_long_pieces(size):
    assert conv_nodes(*size[:4], False) == size[4] and conv_nodes(*size[:4], True) == size[4]


def test_rows_a_thread():
    assert all(conv_step_rows(*s) == 4 for s in CONV_STEP_ROWS)
    assert any(s[0] % 4 for s in CONV_STEP_ROWS)


def test_every_form_of_every_product():
    """Five forms of three products, of pairs (fp32, the square of smaller S and the last product of small P) and of single
    factors; single factors' square has two."""
    seen = set()
    for dtype in (0, 1):
        for size in ORTHO:
            short = (min(size[1:]) + 63) // 64 * 64
            seen |= {(dtype == 0 or short <= (0, 1024, 128)[p], p, f) for p, f in enumerate(ortho_forms(dtype, *size)) if f >= 0}
    assert seen == {(pair, p, f) for pair in (True, False) for p in range(3) for f in range(5)} - {(False, 1, f) for f in (2, 3, 4)}
