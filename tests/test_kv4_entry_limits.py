"""Calls of the 4-bit cache's attention whose grids no launch holds are refused before anything reaches a device."""
import ctypes as C

import pytest

import paper_2406_03853_b200 as eesd
from paper_2406_03853_b200 import binding as b
from tests.test_kv4_entry import AT, UNSUPPORTED, attention, desc, rows, size, tensor


@pytest.mark.parametrize("heads,B,n_rows", [(1 << 26, 1024, 16), (1 << 26, 1024, 15), (1 << 23, 1024, 16), (1 << 24, 256, 16), ((1 << 22) + 2, 1024, 16)])
def test_grids_past_31_bits_are_refused(heads, B, n_rows):
    """segments of eight columns: from 2^31 up to 2^37, some just above 2^32, of which a cut count would leave a small grid"""
    d = desc(heads=1)
    p, n = C.addressof(d), size(d).total_bytes
    r = rows(rows=n_rows, B=B, pages=1, stride=1)
    segments = B * ((heads * n_rows + 7) // 8)
    assert segments >= 1 << 31
    assert eesd.lib().eesd_kv4_attend_scratch_bytes(p, r, heads) == 0
    assert eesd.lib().eesd_kv4_attend(None, p, AT, n, attention(r, 0, tensor(), heads, 0.125, 0, AT, 0, 0)) == UNSUPPORTED


def test_runs_have_a_grid_of_their_own():
    """many segments of long tables are shared out by runs: not refused for their number (no scratch memory is given)"""
    d = desc(heads=1)
    p, n = C.addressof(d), size(d).total_bytes
    r = rows(rows=16, B=1024, pages=512, stride=512)
    need = eesd.lib().eesd_kv4_attend_scratch_bytes(p, r, 1 << 21)
    assert need > 0
    assert eesd.lib().eesd_kv4_attend(None, p, AT, n, attention(r, 0, tensor(), 1 << 21, 0.125, 0, AT, 0, 0)) == -1
