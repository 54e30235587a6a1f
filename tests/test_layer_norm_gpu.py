"""Layer norm and its gradients on the GPU against their formulas in 64 bits.

Tolerances.  A sum of n terms over lanes that add E of them in turn (E <= 64) and then at most 16 partial sums is off by at
most (E + 16) 2^-24 of the sum of the magnitudes; C = 128 bounds that and the few roundings of an expression around it.
Outputs are rounded once more, by half a step of their type."""
import math

import pytest
import torch

import block_reference as ref
from paper_2304_13013_amd import switchback as sb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
C = 128 * 2.0 ** -24

#: one row and one column; widths around every group of waves and every piece; odd ones; the widest
SHAPES = [(1, 1), (3, 7), (5, 8), (2, 64), (197, 768), (64, 513), (33, 1001), (129, 1024), (1000, 1280), (70, 1536), (9, 2047), (13, 2048),
          (31, 2056), (12, 4095), (10, 4104), (7, 8184), (6, 8191), (5, 8193), (9, 12296), (4, 16384), (3, 16392), (2, 16385),
          (2, 65536), (3, 65535)]


def rows_of(b, n, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(b, n, generator=gen) * (0.5 + torch.rand(n, generator=gen)) + 3.0 * torch.randn(b, 1, generator=gen)
    return x.to(dtype), (0.1 * torch.randn(b, n, generator=gen)).to(dtype), 1.0 + 0.3 * torch.randn(n, generator=gen), 0.2 * torch.randn(n, generator=gen)


def on(t):
    return None if t is None else t.to(DEV)


def within(got, want, tol, what):
    off = (got.cpu().double() - want).abs()
    assert torch.isfinite(off).all() and (off <= tol).all(), "%s: off by %g of the tolerance" % (what, float((off / tol).max()))


def check_forward(x, gamma, beta, eps, y, mean, rstd):
    want, mu, r = ref.layer_norm(x, gamma, beta, eps)
    wide = x.double()
    tol_mu = C * wide.abs().mean(1) + 1e-45
    within(mean, mu, tol_mu, "mean")
    # The mean's error enters the variance squared, the sum of squares like every sum.
    within(rstd, r, r * (C + (tol_mu * r) ** 2), "rstd")
    g = 1.0 if gamma is None else gamma.double().abs()
    b = 0.0 if beta is None else beta.double().abs()
    h = ((wide - mu[:, None]) * r[:, None]).abs()
    tol = C * (h * g + b) + g * r[:, None] * tol_mu[:, None] * (1 + C) + g * h * ((tol_mu * r) ** 2)[:, None]
    within(y, want, tol + torch.finfo(x.dtype).eps / 2 * (want.abs() + tol) + 1e-45, "y")


def check_backward(dy, x, mean, rstd, gamma, dx, dgamma, dbeta):
    want, dg, db, h, a = ref.layer_norm_backward(dy, x, mean, rstd, gamma)
    r = rstd.double()[:, None]
    tol = C * r * (a.abs() + a.abs().mean(1, keepdim=True) + 2 * h.abs() * (a * h).abs().mean(1, keepdim=True))
    # x - mean is formed in binary32: half a step of the difference, which h has.
    within(dx, want, tol + torch.finfo(x.dtype).eps / 2 * (want.abs() + tol) + 1e-45, "dx")
    if dgamma is not None:
        terms = (x.shape[0] / 256 + 128) * 2.0 ** -24
        within(dgamma, dg, terms * (dy.double() * h).abs().sum(0) + 1e-45, "dgamma")
        within(dbeta, db, terms * dy.double().abs().sum(0) + 1e-45, "dbeta")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("b,n", SHAPES)
def test_forward_and_backward(b, n, dtype):
    x, dy, gamma, beta = rows_of(b, n, dtype, 7 * b + n)
    y, mean, rstd = sb.layer_norm(on(x), on(gamma), on(beta), eps=1e-5)
    dx, dgamma, dbeta = sb.layer_norm_backward(on(dy), on(x), mean, rstd, on(gamma))
    check_forward(x, gamma, beta, 1e-5, y, mean, rstd)
    check_backward(dy, x, mean.cpu(), rstd.cpu(), gamma, dx, dgamma, dbeta)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [7, 768, 1001, 4096, 8193, 20000])
def test_without_weights(n, dtype):
    """No gamma, no beta, no sums; and the sums without gamma."""
    x, dy, gamma, beta = rows_of(37, n, dtype, n)
    y, mean, rstd = sb.layer_norm(on(x), eps=0.5)
    check_forward(x, None, None, 0.5, y, mean, rstd)
    check_forward(x, gamma, None, 0.5, *sb.layer_norm(on(x), on(gamma), eps=0.5))
    check_forward(x, None, beta, 0.5, *sb.layer_norm(on(x), None, on(beta), eps=0.5))
    dx, none, nothing = sb.layer_norm_backward(on(dy), on(x), mean, rstd, affine=False)
    assert none is None and nothing is None
    check_backward(dy, x, mean.cpu(), rstd.cpu(), None, dx, None, None)
    dx2, dgamma, dbeta = sb.layer_norm_backward(on(dy), on(x), mean, rstd)
    assert torch.equal(dx, dx2)
    check_backward(dy, x, mean.cpu(), rstd.cpu(), None, dx2, dgamma, dbeta)


@pytest.mark.parametrize("b,n", [(512, 2056), (513, 2056), (512, 9000), (513, 9000), (511, 8200), (512, 1001), (514, 12001), (4099, 320), (20000, 72), (5000, 2304), (3000, 9000), (2500, 1003),
                                 (2000, 5), (3000, 13), (5000, 67), (4000, 250), (2049, 12), (1500, 3001), (1100, 8191), (1300, 9001)])
def test_many_rows(b, n):
    """More rows than groups that walk them: a group's registers carry sums from row to row."""
    x, dy, gamma, beta = rows_of(b, n, torch.bfloat16, b + n)
    y, mean, rstd = sb.layer_norm(on(x), on(gamma), on(beta))
    check_forward(x, gamma, beta, 1e-5, y, mean, rstd)
    out = [sb.layer_norm_backward(on(dy), on(x), mean, rstd, on(gamma)) for _ in range(2)]
    check_backward(dy, x, mean.cpu(), rstd.cpu(), gamma, *out[0])
    assert all(torch.equal(p, q) for p, q in zip(*out)), "the same inputs give the same bits"


@pytest.mark.parametrize("b,n", [(2000, 3), (3000, 13), (5000, 66), (4000, 250), (2049, 770), (1500, 3001), (1100, 8191), (1200, 4100)])
def test_many_rows_in_f32(b, n):
    x, dy, gamma, beta = rows_of(b, n, torch.float32, b + n)
    y, mean, rstd = sb.layer_norm(on(x), on(gamma), on(beta))
    check_forward(x, gamma, beta, 1e-5, y, mean, rstd)
    check_backward(dy, x, mean.cpu(), rstd.cpu(), gamma, *sb.layer_norm_backward(on(dy), on(x), mean, rstd, on(gamma)))


def test_no_rows():
    x = torch.empty(0, 96, dtype=torch.bfloat16, device=DEV)
    y, mean, rstd = sb.layer_norm(x)
    assert y.shape == (0, 96) and mean.shape == rstd.shape == (0,)
    dx, dgamma, dbeta = sb.layer_norm_backward(x, x, mean, rstd)
    assert dx.shape == (0, 96) and not dgamma.any() and not dbeta.any()


def test_rows_that_are_constant_large_or_tiny():
    """A variance of zero, rows far from zero (where E x^2 - mu^2 has no digit left), magnitudes near both ends."""
    x = torch.randn(8, 640, generator=torch.Generator().manual_seed(3))
    x[0] = 5.0
    x[1] = 0.0
    x[2] = 1e4 + x[2]
    x[3] *= 1e-30
    x[4] *= 1e17
    check_forward(x, None, None, 1e-5, *sb.layer_norm(on(x)))
    y, mean, rstd = sb.layer_norm(on(x))
    assert (y[0] == 0).all() and (y[1] == 0).all() and mean[0] == 5.0
    # A row with NaN or infinity leaves the others alone.
    x[5, 3], x[6, 100] = math.nan, math.inf
    z, _, _ = sb.layer_norm(on(x))
    assert torch.isnan(z[5]).all() and torch.isnan(z[6]).all() and torch.equal(z[[0, 1, 2, 3, 4, 7]], y[[0, 1, 2, 3, 4, 7]])


def test_outputs_of_the_callers():
    x, dy, gamma, beta = rows_of(50, 264, torch.float32, 1)
    y, mean, rstd = torch.empty(50, 264, device=DEV), torch.empty(50, device=DEV), torch.empty(50, device=DEV)
    got = sb.layer_norm(on(x), on(gamma), on(beta), y=y, mean=mean, rstd=rstd)
    assert [t.data_ptr() for t in got] == [t.data_ptr() for t in (y, mean, rstd)]
    outs = [torch.empty(50, 264, device=DEV), torch.empty(264, device=DEV), torch.empty(264, device=DEV)]
    ws = torch.empty(sb.workspace_bytes(sb.SB_OP_LAYER_NORM_BACKWARD, 50, 264, 0), dtype=torch.uint8, device=DEV)
    got = sb.layer_norm_backward(on(dy), on(x), mean, rstd, on(gamma), dx=outs[0], dgamma=outs[1], dbeta=outs[2], ws=ws)
    assert [t.data_ptr() for t in got] == [t.data_ptr() for t in outs]
    check_backward(dy, x, mean.cpu(), rstd.cpu(), gamma, *got)


def test_gradients_against_differences():
    """d/dt of sum(weights * y) along random directions of x, gamma and beta, by central differences in 64 bits."""
    gen = torch.Generator().manual_seed(5)
    b, n, eps = 6, 40, 1e-5
    x, gamma, beta, dy = (torch.randn(*s, generator=gen) for s in ((b, n), (n,), (n,), (b, n)))
    y, mean, rstd = sb.layer_norm(on(x), on(gamma), on(beta), eps=eps)
    grads = [g.cpu().double() for g in sb.layer_norm_backward(on(dy), on(x), mean, rstd, on(gamma))]
    loss = lambda *v: (ref.layer_norm(v[0], v[1], v[2], eps)[0] * dy.double()).sum()
    at = [t.double() for t in (x, gamma, beta)]
    for i, grad in enumerate(grads):
        along = torch.randn(grad.shape, generator=gen, dtype=torch.float64)
        t = 1e-5
        plus, minus = ([v + s * t * along if j == i else v for j, v in enumerate(at)] for s in (1, -1))
        slope = (loss(*plus) - loss(*minus)) / (2 * t)
        # Differences: t^2 times third derivatives of order one; the gradient's own error: C of its magnitudes.
        assert abs(float((grad * along).sum() - slope)) <= 1e-6 + C * float((grad.abs() * along.abs()).sum()) * 4


def test_captured_in_a_graph():
    x, dy, gamma, beta = (on(t) for t in rows_of(777, 1088, torch.bfloat16, 11))
    bufs = [torch.empty_like(x), torch.empty(777, device=DEV), torch.empty(777, device=DEV), torch.empty_like(x),
            torch.empty(1088, device=DEV), torch.empty(1088, device=DEV)]
    ws = torch.empty(sb.workspace_bytes(sb.SB_OP_LAYER_NORM_BACKWARD, 777, 1088, 0), dtype=torch.uint8, device=DEV)

    def step():
        sb.layer_norm(x, gamma, beta, y=bufs[0], mean=bufs[1], rstd=bufs[2])
        sb.layer_norm_backward(dy, x, bufs[1], bufs[2], gamma, dx=bufs[3], dgamma=bufs[4], dbeta=bufs[5], ws=ws)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for i in range(3):
        x.copy_(torch.randn_like(x))
        dy.copy_(torch.randn_like(dy))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in bufs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(replayed, bufs)), "replay %d" % i


def test_rows_behind_four_gib():
    """The last of 2.6e9 elements: their results are those of the last rows alone."""
    b, n, last = 640000, 4096, 700
    x = torch.randn(b, n, dtype=torch.bfloat16, device=DEV, generator=torch.Generator(device=DEV).manual_seed(6))
    gamma, beta = torch.rand(n, device=DEV), torch.rand(n, device=DEV)
    y, mean, rstd = sb.layer_norm(x, gamma, beta)
    end = sb.layer_norm(x[-last:], gamma, beta)
    assert all(torch.equal(p[-last:], q) for p, q in zip((y, mean, rstd), end))
    y.zero_()  # dy of all rows but the last ones: dgamma and dbeta are theirs
    dy = y
    dy[-last:] = x[:last]
    dx, dgamma, dbeta = sb.layer_norm_backward(dy, x, mean, rstd, gamma)
    assert not dx[:-last].any()
    check_backward(dy[-last:].cpu(), x[-last:].cpu(), mean[-last:].cpu(), rstd[-last:].cpu(), gamma.cpu(), dx[-last:], dgamma, dbeta)
