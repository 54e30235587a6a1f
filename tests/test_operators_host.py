"""What the layer norm and the block-scaled float8 calls refuse, on the host: nothing is launched, no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2304_13013_amd import switchback as sb

INVALID, SHAPE, WS = 1, 2, 3
FAKE, ODD, NULL = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004), ctypes.c_void_p(None)  # never dereferenced


@pytest.fixture(scope="module")
def lib():
    return sb.load_library()


def test_layer_norm_refuses(lib):
    def norm(x=FAKE, dtype=0, gamma=FAKE, beta=FAKE, eps=1e-5, rows=4, cols=64, y=FAKE, mean=FAKE, rstd=FAKE):
        return lib.switchback_layer_norm(x, dtype, gamma, beta, eps, rows, cols, y, mean, rstd, NULL)
    assert norm(dtype=2) == norm(dtype=7) == norm(rows=-1) == norm(cols=0) == INVALID
    assert norm(eps=0.0) == norm(eps=-1.0) == norm(eps=float("nan")) == norm(eps=float("inf")) == INVALID
    assert norm(x=NULL) == norm(y=NULL) == norm(x=ODD) == norm(y=ODD) == norm(gamma=ODD) == norm(beta=ODD) == INVALID
    assert norm(mean=ctypes.c_void_p(0x1002)) == norm(rstd=ctypes.c_void_p(0x1001)) == INVALID
    assert norm(cols=65537) == norm(rows=(1 << 30) + 1) == SHAPE
    assert norm(rows=0, x=NULL, y=NULL) == 0

    def back(dy=FAKE, x=FAKE, dtype=1, mean=FAKE, rstd=FAKE, gamma=FAKE, rows=4000, cols=64, dx=FAKE, dgamma=FAKE, dbeta=FAKE, ws=FAKE, size=1 << 30):
        return lib.switchback_layer_norm_backward(dy, x, dtype, mean, rstd, gamma, rows, cols, dx, dgamma, dbeta, ws, size, NULL)
    assert back(dtype=2) == back(rows=-1) == back(cols=0) == INVALID
    for name in ("dy", "x", "mean", "rstd", "dx", "ws"):
        assert back(**{name: NULL}) == INVALID, name
    for name in ("dy", "x", "gamma", "dx", "ws"):
        assert back(**{name: ODD}) == INVALID, name
    assert back(cols=65537) == back(rows=(1 << 30) + 1) == SHAPE
    assert back(size=sb.workspace_bytes(sb.SB_OP_LAYER_NORM_BACKWARD, 4000, 64, 0) - 1) == WS
    assert sb.workspace_bytes(sb.SB_OP_LAYER_NORM_BACKWARD, 0, 64, 0) == sb.workspace_bytes(sb.SB_OP_LAYER_NORM_BACKWARD, 4, 64, 0) == sb.workspace_bytes(sb.SB_OP_LAYER_NORM_BACKWARD, 4, 1 << 20, 0) == 0


def test_block_calls_refuse(lib):
    def rows(x=FAKE, rows=4, cols=64, fmt=0, codes=FAKE, scales=FAKE):
        return lib.switchback_quantize_rowwise_f8_block(x, rows, cols, fmt, codes, scales, NULL)
    assert rows(fmt=2) == rows(rows=-1) == rows(cols=0) == rows(x=NULL) == rows(codes=ODD) == rows(scales=ODD) == INVALID
    assert rows(cols=60) == rows(cols=131080) == rows(rows=(1 << 30) + 1) == SHAPE
    assert rows(rows=0, x=NULL, codes=NULL, scales=NULL) == 0

    def weight(w=FAKE, experts=1, m=64, n=64, fmt=0, codes=FAKE, scales=FAKE, codes_t=FAKE, scales_t=FAKE):
        return lib.switchback_quantize_weight_f8_block(w, experts, m, n, fmt, codes, scales, codes_t, scales_t, NULL)
    assert weight(fmt=5) == weight(experts=0) == weight(m=0) == weight(n=-64) == INVALID
    assert weight(w=NULL) == weight(codes=ODD) == weight(codes_t=NULL) == weight(scales_t=NULL) == weight(scales_t=ODD) == INVALID
    assert weight(m=96) == weight(n=8) == weight(experts=1025) == weight(m=65536, n=65536) == SHAPE

    def product(a=FAKE, fa=0, sa=FAKE, b=FAKE, fb=0, sb_=FAKE, offsets=NULL, experts=1, M=4, N=64, K=128, out=FAKE, dtype=0):
        return lib.switchback_matmul_f8_block(a, fa, sa, b, fb, sb_, offsets, experts, M, N, K, out, dtype, NULL)
    assert product(fa=2) == product(fb=-1) == product(dtype=2) == product(M=-1) == product(N=0) == product(K=0) == INVALID
    assert product(experts=2) == product(experts=0, offsets=FAKE) == product(offsets=ctypes.c_void_p(0x1002)) == INVALID
    for name in ("a", "sa", "b", "sb_", "out"):
        assert product(**{name: NULL}) == product(**{name: ODD}) == INVALID, name
    assert product(K=64) == product(N=32) == product(K=131072 + 128) == product(experts=1025, offsets=FAKE) == SHAPE
    assert product(M=1 << 24, N=128, K=128) == product(M=128, N=32768, K=131072) == SHAPE  # 32-bit offsets into rows, into a weight
    assert product(M=0, a=NULL, out=NULL) == 0

    def linear(x=FAKE, w=FAKE, sw=FAKE, offsets=NULL, experts=1, b=4, n=64, m=64, fx=0, fw=0, y=FAKE, dtype=0, ws=FAKE, size=1 << 30):
        return lib.switchback_linear_f8_block(x, w, sw, offsets, experts, b, n, m, fx, fw, y, dtype, ws, size, NULL)
    assert linear(fx=2) == linear(fw=2) == linear(dtype=2) == linear(b=-1) == linear(experts=3) == INVALID
    for name in ("x", "w", "sw", "y"):
        assert linear(**{name: NULL}) == linear(**{name: ODD}) == INVALID, name
    assert linear(n=96) == linear(m=32) == SHAPE
    need = lib.switchback_linear_f8_block_workspace_bytes(4000, 1024, 1024, 1)
    assert need == sb.workspace_bytes(sb.SB_OP_FORWARD_F8_BLOCK, 4000, 1024, 0) and lib.switchback_linear_f8_block_workspace_bytes(4, 64, 64, 1) == 0
    assert linear(b=4000, n=1024, m=1024, size=need - 1) == WS and linear(b=4000, n=1024, m=1024, ws=NULL) == INVALID
    assert linear(b=4000, n=1024, m=1024, ws=ODD) == INVALID
    assert linear(b=0, x=NULL, y=NULL, ws=NULL, size=0) == 0

    def forward(x=FAKE, w=FAKE, offsets=NULL, experts=1, b=4, n=64, m=64, fx=0, fw=0, wq=FAKE, sw=FAKE, wt=FAKE, st=FAKE, y=FAKE, dtype=0,
                ws=FAKE, size=1 << 30):
        return lib.switchback_forward_f8_block(x, w, offsets, experts, b, n, m, fx, fw, wq, sw, wt, st, y, dtype, ws, size, NULL)
    assert forward(fx=2) == forward(fw=2) == forward(dtype=2) == forward(experts=3) == forward(wt=NULL) == forward(st=NULL) == INVALID
    for name in ("x", "w", "wq", "sw", "y", "ws"):
        assert forward(**{name: NULL}) == forward(**{name: ODD}) == INVALID, name
    assert forward(n=100) == forward(m=32) == SHAPE and forward(size=8) == WS

    def gradient(dy=FAKE, x=FAKE, offsets=FAKE, experts=2, b=4, n=64, m=64, dw=FAKE, dtype=0, ws=FAKE, size=1 << 40):
        return lib.switchback_backward_weight_experts(dy, x, offsets, experts, b, n, m, dw, dtype, ws, size, NULL)
    assert gradient(dtype=2) == gradient(offsets=NULL) == gradient(experts=0) == gradient(b=-1) == INVALID
    assert gradient(dy=NULL) == gradient(x=ODD) == gradient(dw=ODD) == gradient(offsets=ctypes.c_void_p(0x1002)) == INVALID
    assert gradient(n=96) == gradient(m=32) == gradient(experts=1025) == SHAPE
    need = lib.switchback_backward_weight_experts_workspace_bytes(20000, 256, 256, 2)
    assert need > 0 and gradient(b=20000, n=256, m=256, size=need - 1) == WS
    assert gradient(b=20000, n=256, m=256, ws=NULL) == INVALID
    assert lib.switchback_backward_weight_experts_workspace_bytes(100, 96, 64, 2) == 0


def test_binding_refuses():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    where = torch.zeros(3, dtype=torch.int32)
    refused = [
        lambda: sb.layer_norm(bf(4, 64)), lambda: sb.layer_norm(torch.zeros(4, 64, dtype=torch.float16)),
        lambda: sb.layer_norm(torch.zeros(4, 64, dtype=torch.float64)), lambda: sb.layer_norm(bf(4, 64), torch.ones(32)),
        lambda: sb.layer_norm(bf(4, 64), y=bf(4, 32)), lambda: sb.layer_norm(bf(4, 64), torch.ones(64, dtype=torch.bfloat16)),
        lambda: sb.layer_norm_backward(bf(4, 64), torch.zeros(4, 64), torch.zeros(4), torch.zeros(4)),
        lambda: sb.layer_norm_backward(bf(4, 32), bf(4, 64), torch.zeros(4), torch.zeros(4)),
        lambda: sb.layer_norm_backward(bf(4, 64), bf(4, 64), torch.zeros(3), torch.zeros(4)),
        lambda: sb.layer_norm_backward(bf(4, 64), bf(4, 64), torch.zeros(4), torch.zeros(4), affine=False, dgamma=torch.zeros(64)),
        lambda: sb.quantize_rowwise_f8_block(bf(4, 64), 0), lambda: sb.quantize_rowwise_f8_block(bf(4, 64), 0, codes=u8(4, 64)),
        lambda: sb.quantize_rowwise_f8_block(bf(4, 64), 0, scales=u8(4, 4)), lambda: sb.quantize_weight_f8_block(bf(64), 0),
        lambda: sb.quantize_weight_f8_block(bf(64, 64), 0, codes_t=u8(64, 64)), lambda: sb.quantize_weight_f8_block(bf(2, 2, 64, 64), 0),
        lambda: sb.matmul_f8_block(u8(4, 128), 0, u8(1, 4, 4), u8(64, 256), 0, u8(1, 2)),
        lambda: sb.matmul_f8_block(u8(4, 128), 0, u8(1, 4, 4), u8(64, 128), 0, u8(1, 1), offsets=where),
        lambda: sb.matmul_f8_block(u8(4, 128), 0, u8(1, 4, 4), u8(2, 64, 128), 0, u8(2, 1, 1)),
        lambda: sb.matmul_f8_block(u8(4, 128), 0, u8(1, 4, 4), u8(3, 64, 128), 0, u8(3, 1, 1), offsets=where),
        lambda: sb.matmul_f8_block(u8(4, 128), 0, u8(4, 4), u8(64, 128), 0, u8(1, 1)),
        lambda: sb.matmul_f8_block(u8(4, 128), 0, u8(1, 4, 4), u8(64, 128), 0, u8(1, 2)),
        lambda: sb.matmul_f8_block(u8(4, 128), 0, u8(1, 4, 4), u8(64, 128), 0, u8(1, 1), out=torch.zeros(4, 64, dtype=torch.int32)),
        lambda: sb.linear_f8_block(bf(4, 64), u8(64, 64), u8(1, 1)), lambda: sb.linear_f8_block(bf(4, 64), u8(64, 128), u8(1, 1), y=bf(4, 32)),
        lambda: sb.linear_f8_block(bf(4, 64), u8(64, 128), u8(1, 1), y=torch.zeros(4, 64, dtype=torch.float16)),
        lambda: sb.forward_f8_block(bf(4, 64), bf(64, 128)), lambda: sb.forward_f8_block(bf(4, 64), bf(2, 64, 64), sb.BlockBuffers(4, 64, 64, 2, "cpu")),
        lambda: sb.forward_f8_block(bf(4, 64), bf(2, 64, 64), sb.BlockBuffers(4, 64, 64, None, "cpu"), offsets=where),
        lambda: sb.forward_f8_block(bf(4, 64), bf(64, 64), sb.BlockBuffers(5, 64, 64, None, "cpu")),
        lambda: sb.backward_input_f8_block(bf(4, 128), sb.BlockBuffers(4, 64, 64, None, "cpu")),
        lambda: sb.backward_input_f8_block(bf(4, 64), sb.BlockBuffers(4, 64, 64, 2, "cpu")),
        lambda: sb.backward_weight_experts(bf(4, 64), bf(5, 64), where), lambda: sb.backward_weight_experts(bf(4, 64), bf(4, 64), where.long()),
        lambda: sb.backward_weight_experts(bf(4, 64), bf(4, 64), where, sb.BlockBuffers(4, 64, 64, 3, "cpu")),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(sb.SwitchBackError):
            call()
            pytest.fail("call %d was not refused" % i)


def test_tensors_of_another_gpu_are_refused(monkeypatch):
    """The calls enqueue on the current device's stream."""
    class Elsewhere:
        def __init__(self, device):
            self.device = device

        def get_device(self):
            return self.device

    monkeypatch.setattr(sb, "_current_device", lambda: 0)
    sb._on_current_device(Elsewhere(0), None, Elsewhere(-1))
    with pytest.raises(sb.SwitchBackError):
        sb._on_current_device(Elsewhere(0), Elsewhere(1))


def test_workspaces(lib):
    assert sb.workspace_bytes(sb.SB_OP_FORWARD_F8_BLOCK, 100, 64, 0) == 100 * 128 + 100 * 4       # codes of whole blocks, a dword of scales a row
    assert sb.workspace_bytes(sb.SB_OP_FORWARD_F8_BLOCK, 3, 1088, 0) == -(-3 * 1152 // 256) * 256 + 3 * 12
    bufs = sb.BlockBuffers(7, 192, 320, 3, "cpu")
    assert tuple(bufs.wq.shape) == (3, 320, 256) and tuple(bufs.wq_t.shape) == (3, 192, 384)
    assert tuple(bufs.scales_w.shape) == (3, 3, 2) and tuple(bufs.scales_wt.shape) == (3, 2, 3)
    assert bufs.ws.numel() >= sb.workspace_bytes(sb.SB_OP_FORWARD_F8_BLOCK, 7, 192, 0)
    big = sb.BlockBuffers(4000, 192, 2048, None, "cpu")
    assert big.ws.numel() >= sb.workspace_bytes(sb.SB_OP_FORWARD_F8_BLOCK, 4000, 2048, 0) == lib.switchback_linear_f8_block_workspace_bytes(4000, 2048, 192, 1)


def test_memory_in_common_is_refused(lib):
    """A row that is written while others are still read: the calls that allow no output over an input say so."""
    at = lambda i: ctypes.c_void_p(0x100000 + i)  # never dereferenced
    far = at(1 << 20)
    norm = lambda x, y: lib.switchback_layer_norm(x, 0, NULL, NULL, 1e-5, 4, 64, y, NULL, NULL, NULL)
    back = lambda dy, x, dx: lib.switchback_layer_norm_backward(dy, x, 1, FAKE, FAKE, NULL, 4, 64, dx, NULL, NULL, NULL, 0, NULL)
    assert norm(at(0), at(0)) == norm(at(0), at(4 * 64 * 2 - 16)) == norm(at(16), at(0)) == INVALID
    assert back(at(0), far, at(0)) == back(far, at(0), at(4 * 64 * 4 - 16)) == back(at(16), far, at(0)) == INVALID

    def linear(x, y, dtype, b=4, m=128):
        return lib.switchback_linear_f8_block(x, FAKE, FAKE, NULL, 1, b, 64, m, 0, 0, y, dtype, far, 1 << 30, NULL)
    assert linear(at(0), at(0), 0) == linear(at(0), at(4 * 64 * 2 - 16), 0) == linear(at(4 * 128 * 4 - 16), at(0), 1) == INVALID
    assert linear(at(0), at(0), 0, 4000, 2048) == INVALID


def test_workspaces_of_the_callers_lie_on_the_gpu():
    for ws in (torch.zeros(64, dtype=torch.uint8), torch.zeros(64)):
        with pytest.raises(sb.SwitchBackError):
            sb._given_ws(ws)
    assert sb._given_ws(None) == (None, 0)
    with pytest.raises(sb.SwitchBackError):
        sb.backward_weight_experts(torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(0, dtype=torch.int32))


def test_most_rows_of_a_launch(lib):
    """A workgroup for 16 rows of 512 columns: a launch has fewer than 2^32 threads."""
    rows = lambda rows, cols: lib.switchback_quantize_rowwise_f8_block(FAKE, rows, cols, 0, FAKE, FAKE, NULL)
    assert rows((1 << 27) + 1, 8) == rows(1 << 26, 1032) == rows(1 << 20, 131072) == SHAPE
