"""Weight gradients of experts that get most of the tokens, on the GPU: how long their sums' chains of additions are.

A chain of K additions of terms with random signs, each with a uniform error of at most half a step of a partial sum that grows with
the root of its place, ends with a relative error of 2^-24 / 3^1/2 * (K / 2)^1/2; the matrix instruction adds 16 products at a time,
so K is T / 16 for T tokens: 3.9e-7 at 4096.  Pieces of random errors leave their sum with the relative error of one, and
each addition of pieces adds less than 2^-24 / 3^1/2."""
import pytest
import torch

from paper_2304_13013_amd import switchback as sb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def chain_error(tokens):
    return 2.0 ** -24 / 3 ** 0.5 * (tokens / 32) ** 0.5


def relative_error(got, want):
    return float((got.double() - want).square().mean().sqrt() / want.square().mean().sqrt())


@pytest.mark.parametrize("n,m,experts,tokens,at", [(1024, 4096, 8, 16448, 3), (256, 320, 2, 200000, 0), (320, 576, 64, 16384, 63),
                                                   (1280, 2560, 2, 65536, 1), (64, 64, 16, 150000, 5), (1088, 768, 32, 6080, 0),
                                                   (1088, 768, 32, 6081, 1), (2048, 1088, 5, 10240, 4)],
                         ids=["whole", "split", "small", "few", "tiny", "one piece", "two pieces", "wide"])
def test_gradient_of_a_long_expert(n, m, experts, tokens, at):
    """All rows on one of the experts: no chain has more than 95 stages of 64 tokens, whatever the routing.  (In one chain 16384
    tokens are off by 8e-7.)"""
    gen = torch.Generator(device=DEV).manual_seed(n)
    dy, x = (torch.randn(tokens, k, generator=gen, device=DEV).bfloat16() for k in (m, n))
    where = torch.tensor([0] * (at + 1) + [tokens] * (experts - at), dtype=torch.int32, device=DEV)
    dw = sb.backward_weight_experts(dy, x, where, dw_dtype=torch.float32)
    assert not dw[:at].any() and not dw[at + 1:].any()
    assert torch.equal(sb.backward_weight_experts(dy, x, where, dw_dtype=torch.bfloat16), dw.bfloat16())
    error = relative_error(dw[at], dy.double().t().contiguous() @ x.double())
    bound = 1.05 * (chain_error(95 * 64) ** 2 + (tokens / 4096) * 2.0 ** -48 / 3) ** 0.5
    assert error <= bound, "%g, bound %g" % (error, bound)


def test_gradient_of_a_long_expert_against_the_plain_one():
    """16448 tokens, 1024 -> 4096, all of one of eight experts: no further from 64 bits than the plain layer's gradient, which
    sums them in four pieces."""
    tokens, n, m = 16448, 1024, 4096
    gen = torch.Generator(device=DEV).manual_seed(1)
    dy, x = (torch.randn(tokens, k, generator=gen, device=DEV).bfloat16() for k in (m, n))
    want = dy.double().t().contiguous() @ x.double()
    where = torch.tensor([0] * 3 + [tokens] * 6, dtype=torch.int32, device=DEV)
    plain = relative_error(sb.backward_weight(dy, x, dw_dtype=torch.float32), want)
    assert relative_error(sb.backward_weight_experts(dy, x, where, dw_dtype=torch.float32)[2], want) <= 1.1 * plain


@pytest.mark.parametrize("n,m,experts", [(1024, 4096, 6), (512, 1024, 16)], ids=["wide", "small"])
def test_pieces_of_uneven_experts_in_a_graph(n, m, experts):
    """Experts of one and of several pieces, replayed with other rows and other offsets: the eager results every time, and close to
    64 bits."""
    b = 24000
    gen = torch.Generator(device=DEV).manual_seed(3)
    dy, x = (torch.zeros(b, k, dtype=torch.bfloat16, device=DEV) for k in (m, n))
    where = torch.zeros(experts + 1, dtype=torch.int32, device=DEV)
    need = sb._experts_workspace(b, n, m, experts, DEV).numel()
    bufs = sb.BlockBuffers(b, n, m, experts)
    assert bufs.ws_dw.numel() == need
    dw = torch.zeros(experts, m, n, device=DEV)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        sb.backward_weight_experts(dy, x, where, bufs, dw=dw)
    for counts in ([100, 0, 20000, 64, 6080, 1000], [24000, 0, 0, 0, 0, 0], [6081, 6144, 6145, 4100, 0, 1], [0, 0, 0, 0, 0, 23999]):
        dy.copy_(torch.randn(b, m, generator=gen, device=DEV))
        x.copy_(torch.randn(b, n, generator=gen, device=DEV))
        counts = counts[:5] + [0] * (experts - 6) + [counts[5]]
        where.copy_(torch.tensor([sum(counts[:e]) for e in range(experts + 1)], dtype=torch.int32))
        bufs.ws_dw.fill_(255)  # NaN, wherever it is read before it is written
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, sb.backward_weight_experts(dy, x, where, dw_dtype=torch.float32)), counts
        for e, count in enumerate(counts):
            rows = slice(int(where[e]), int(where[e]) + count)
            want = dy[rows].double().t().contiguous() @ x[rows].double()
            assert float((dw[e].double() - want).norm()) <= 1e-6 * float(want.norm()) + 1e-30, (counts, e)
