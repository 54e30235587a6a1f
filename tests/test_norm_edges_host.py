"""Layer norm's workspace on the host: what its gradients ask for, and no more."""
from paper_2304_13013_amd import switchback as sb


def test_workspace_of_wide_rows():
    need = lambda rows, cols: sb.workspace_bytes(sb.SB_OP_LAYER_NORM_BACKWARD, rows, cols, 0)
    # Few rows that fit in a workgroup: one launch, no workspace, in either type.
    assert need(4, 12288) == need(1, 16384) == need(256, 9000) == need(4, 8191) == need(1024, 4096) == 0
    # Where one type's rows are no whole pieces, they may not fit, and a row's terms are a pair of vectors of their own.
    assert need(4, 8193) == 4 * 2 * 8193 * 4 and need(4, 9004) == 4 * 2 * 9004 * 4
    assert need(3, 16392) == 3 * 2 * 16392 * 4 and need(1, 65536) == 2 * 65536 * 4
    assert need(256, 20000) == need(100000, 20000) == 256 * 2 * 20000 * 4
