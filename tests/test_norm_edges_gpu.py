"""Layer norm at the edges of what it allows, on the GPU: rows far from zero, rows that start anywhere, the widest rows."""
import pytest
import torch

import block_reference as ref
from paper_2304_13013_amd import switchback as sb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPE = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])


@TYPE
@pytest.mark.parametrize("n", [100, 640, 1088, 1280, 1920, 2047, 4100, 8191, 8193, 12296, 16388, 30000, 65535])
def test_norm_of_rows_far_from_zero(n, dtype):
    """Constant rows give zeros, and rows of a few steps around a large value what these steps give.

    Tolerances.  A first mean is off by at most C |mu| (C = 128 * 2^-24, sums over lanes and waves).  Differences from it are exact
    (both lie within a factor of two), of size S + C |mu| with S the row's largest distance from its mean, and their mean c is off
    by C times that; so are the differences less c, and y by r times it.  The variance is the mean of their squares less c^2,
    off by 4 C (S + C |mu|)^2."""
    C = 128 * 2.0 ** -24
    gen = torch.Generator().manual_seed(n)
    x = torch.empty(7, n)
    for i, value in enumerate((1000.0, 10000.0, 777.77, -1e5)):
        x[i] = value
    for i, value in enumerate((1000.0, 10000.0, -777.0)):
        x[4 + i] = value + (8.0 if dtype == torch.bfloat16 else 2.0 ** -9) * torch.randint(-3, 4, (n,), generator=gen)
    x = x.to(dtype)
    y, mean, rstd = (t.cpu().double() for t in sb.layer_norm(x.to(DEV), eps=1e-5))
    want, mu, r = ref.layer_norm(x, None, None, 1e-5)
    size = (x.double() - mu[:, None]).abs().amax(1) + C * mu.abs()
    assert ((mean - mu).abs() <= 2.0 ** -24 * mu.abs() + 2 * C * size).all(), "mean"
    tol_r = C + 4 * C * size ** 2 * r ** 2
    assert ((rstd - r).abs() <= tol_r * r).all(), "rstd"
    tol = 2 * C * (size * r)[:, None] + want.abs() * tol_r[:, None]
    off = (y - want).abs()
    assert (off <= tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol)).all(), "y off by %g" % float(off.max())


@TYPE
@pytest.mark.parametrize("b,n", [(4, 12288), (1, 16384), (64, 9000), (3, 16392), (4, 65536), (300, 16388)])
def test_norm_gradients_in_the_workspace_asked_for(b, n, dtype):
    """No more than the call asks for, and none where it asks for none."""
    gen = torch.Generator().manual_seed(b + n)
    x, dy = (torch.randn(b, n, generator=gen).to(dtype) for _ in range(2))
    need = sb.workspace_bytes(sb.SB_OP_LAYER_NORM_BACKWARD, b, n, 0)
    mean, rstd = torch.zeros(b, device=DEV), torch.ones(b, device=DEV)
    store = torch.full((need + 4096,), 77, dtype=torch.uint8, device=DEV)
    dx, dgamma, dbeta = sb.layer_norm_backward(dy.to(DEV), x.to(DEV), mean, rstd, ws=store[:need] if need else None)
    assert (store[need:] == 77).all()
    want = ref.layer_norm_backward(dy, x, mean.cpu(), rstd.cpu(), None)
    for got, wide, size in ((dgamma, want[1], (dy.double() * x.double()).abs().sum(0)), (dbeta, want[2], dy.double().abs().sum(0))):
        assert ((got.cpu().double() - wide).abs() <= (b / 256 + 128) * 2.0 ** -24 * size).all()


@TYPE
@pytest.mark.parametrize("b,n", [(6, 3), (6, 7), (9, 13), (40, 1001), (5, 8191), (4, 8193), (1500, 67)])
def test_norm_of_rows_that_start_anywhere(b, n, dtype):
    """Rows that are no whole 16-byte pieces need not start at one: views from the second row on, and outputs in such views."""
    gen = torch.Generator().manual_seed(b + n)
    x, dy = (torch.randn(b + 1, n, generator=gen).to(dtype).to(DEV) for _ in range(2))
    gamma, beta = torch.rand(n, generator=gen).to(DEV), torch.rand(n, generator=gen).to(DEV)
    want = sb.layer_norm(x[1:].clone(), gamma, beta)
    y, dx = torch.full_like(x, -3.0), torch.full_like(x, -3.0)
    got = sb.layer_norm(x[1:], gamma, beta, y=y[1:])
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and (y[0] == -3.0).all()
    back = sb.layer_norm_backward(dy[1:].clone(), x[1:].clone(), want[1], want[2], gamma)
    got = sb.layer_norm_backward(dy[1:], x[1:], want[1], want[2], gamma, dx=dx[1:])
    assert all(torch.equal(p, q) for p, q in zip(got, back)) and (dx[0] == -3.0).all()
