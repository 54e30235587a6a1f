"""Layer norm's workspace and alignment on the host: what its calls ask for, and no more."""
import ctypes

import pytest

from paper_2304_13013_amd import switchback as sb


@pytest.fixture(scope="module")
def lib():
    return sb.load_library()


def test_workspace_of_wide_rows():
    need = lambda rows, cols: sb.workspace_bytes(sb.SB_OP_LAYER_NORM_BACKWARD, rows, cols, 0)
    # Few rows that fit in a workgroup: one launch, no workspace, in either type.
    assert need(4, 12288) == need(1, 16384) == need(256, 9000) == need(4, 8191) == need(1024, 4096) == 0
    # Where one type's rows are no whole pieces, they may not fit, and a row's terms are a pair of vectors of their own.
    assert need(4, 8193) == 4 * 2 * 8193 * 4 and need(4, 9004) == 4 * 2 * 9004 * 4
    assert need(3, 16392) == 3 * 2 * 16392 * 4 and need(1, 65536) == 2 * 65536 * 4
    assert need(256, 20000) == need(100000, 20000) == 256 * 2 * 20000 * 4


def test_rows_start_at_an_element(lib):
    at = ctypes.c_void_p  # never dereferenced
    good, null = at(0x1000), at(None)
    norm = lambda x, y, dtype, cols: lib.switchback_layer_norm(x, dtype, null, null, 1e-5, 4, cols, y, null, null, null)
    back = lambda dy, x, dx, dtype, cols: lib.switchback_layer_norm_backward(dy, x, dtype, good, good, null, 4, cols, dx, null, null, null, 0, null)
    for dtype, odd in ((0, 0x100001), (1, 0x100002)):
        assert norm(at(odd), good, dtype, 63) == norm(good, at(odd), dtype, 63) == 1
        assert back(at(odd), good, good, dtype, 63) == back(good, at(odd), good, dtype, 63) == back(good, good, at(odd), dtype, 63) == 1
    for dtype, cols in ((0, 64), (1, 60)):
        assert norm(at(0x100008), good, dtype, cols) == back(good, at(0x100008), good, dtype, cols) == 1
