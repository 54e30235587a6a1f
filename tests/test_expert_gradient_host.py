"""Plans of the experts' weight gradients on the host: the workspace for sums in pieces."""
from paper_2304_13013_amd import switchback as sb


def test_workspace_of_pieces():
    """A tile of 256 x 256 binary32 values a workgroup where an item may have 96 stages of 64 tokens, and 256x256 tiles run."""
    need = sb.load_library().switchback_backward_weight_experts_workspace_bytes
    tile = 256 * 256 * 4
    assert need(16448, 1024, 4096, 8) == need(6081, 1024, 4096, 8) == 256 * tile
    assert need(10240, 2048, 1088, 5) == 200 * tile  # as many as there are items
    assert need(6080, 1024, 4096, 8) == need(5003, 768, 1088, 24) == 0
    assert need(16384, 320, 576, 64) == 0  # 128x128 tiles keep the sum of the pieces in registers
    assert need(65536, 1280, 2560, 2) == 5 * 2 * 1280 * 2560 * 4 + 256 * tile  # of a split
