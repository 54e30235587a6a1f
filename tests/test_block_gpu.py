"""The float8 layer with a scale for each block of 128, plain and by experts, on the GPU against its definition in 64 bits.

Tolerances.  Codes and scale bytes: equal.  Products: the matrix instruction adds eight neighbouring products after dropping
what lies 2^-13 below the largest of them (seven of them at most), and its sums and those of the waves' pieces are roundings to
binary32: (7 2^-13 + (K / 64 + 8) 2^-23) of the sum of the magnitudes; codes without more than one binary digit lose nothing
and are compared for equality.  Weight gradients: products of two bf16 are exact in binary32, a sum of b of them is off by at
most (b / 32 + 64) 2^-23 of the magnitudes (32 products are one instruction's sum).  Outputs are rounded once more."""
import pytest
import torch

import block_reference as ref
from paper_2304_13013_amd import switchback as sb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E4M3, E5M2 = sb.SB_E4M3, sb.SB_E5M2
FMT = pytest.mark.parametrize("fmt", [E4M3, E5M2], ids=["e4m3", "e5m2"])


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def within(got, want, tol, what):
    # A rounding: half a step relative to the value, below the smallest normal number half of the smallest subnormal (bf16: 2^-126
    # has steps of 2^-133).
    rounding = half_step(got.dtype) * (want.abs() + tol).clamp(min=torch.finfo(got.dtype).smallest_normal)
    tol = tol + rounding + 1e-45
    off = (got.cpu().double() - want).abs()
    assert torch.isfinite(off).all() and (off <= tol).all(), "%s: off by %g of the tolerance" % (what, float((off / tol).max()))


def product_tol(size, k):
    return (7 * 2.0 ** -13 + (k / 64 + 8) * 2.0 ** -23) * size


def row_scales(e):
    """Scale bytes of exponents [rows, blocks] as the kernels take them, [parts, rows, 4], 0 behind the last block."""
    rows, blocks = e.shape
    bytes4 = torch.zeros(rows, -(-blocks // 4), 4, dtype=torch.uint8)
    bytes4.view(rows, -1)[:, :blocks] = e + 127
    return bytes4.transpose(0, 1).contiguous()


def edge_rows(x):
    """Rows (or parts of them) where a scale or a rounding can go wrong."""
    for i in range(min(x.shape[0], 9)):
        row = x[i]
        n = min(x.shape[1], 128)
        if i == 0:
            row[:n] = 0.0                                   # a block without a value
        elif i == 1:
            row[0] = 3.3895313892515355e38                  # the largest bf16
        elif i == 2:
            row[:n] = row[:n] * 2.0 ** -126 * 2.0 ** -5     # subnormals
        elif i == 3:
            row[:n] = row[:n].clamp(-1, 1)
            row[1] = 1.75                                   # 448 and 57344 times a power of two: the scale's last fitting value
        elif i == 4:
            row[:n] = row[:n].clamp(-1, 1)
            row[1] = 1.7578125                              # the next bf16
        elif i == 5:
            row[:n] = (torch.arange(n) - n // 2) / 16.0     # ties
            row[0] = -1.75
        elif i == 6:
            row[:] = 0.0
            row[-1] = -2.0 ** -133                          # the smallest bf16
        elif i == 7:
            row[:n] = 2.0 ** -10 * torch.randn(n)           # the format's subnormals
            row[2] = 400.0
        elif i == 8:
            row[:] = -0.0
    return x


@FMT
@pytest.mark.parametrize("rows,cols", [(1, 8), (3, 64), (17, 128), (16, 136), (300, 520), (33, 1088), (1025, 1280), (5, 8200), (2, 131072)])
def test_row_codes(rows, cols, fmt):
    gen = torch.Generator().manual_seed(rows + cols)
    x = edge_rows((torch.randn(rows, cols, generator=gen) * 3.0).bfloat16())
    codes, scales = sb.quantize_rowwise_f8_block(x.to(DEV), fmt)
    want, e = ref.quantize_rows(x, fmt)
    assert codes.shape == want.shape
    assert torch.equal(ref.decode(codes, fmt), want) and torch.equal(scales.cpu(), row_scales(e))


@FMT
@pytest.mark.parametrize("experts,m,n", [(None, 64, 64), (None, 128, 192), (1, 192, 64), (3, 320, 1088), (None, 1024, 256), (5, 64, 128)])
def test_weight_codes(experts, m, n, fmt):
    gen = torch.Generator().manual_seed(m + n)
    w = (torch.randn(experts or 1, m, n, generator=gen) * 0.05).bfloat16()
    for part in w:
        edge_rows(part[:9])
    w[-1, -64:, -64:] = 0.0
    given = w[0] if experts is None else w
    out = [t.cpu() for t in sb.quantize_weight_f8_block(given.to(DEV), fmt)]
    codes, scales, codes_t, scales_t = [t[None] if experts is None else t for t in out]
    for e in range(experts or 1):
        for c, s, part in ((codes, scales, w[e]), (codes_t, scales_t, w[e].t())):
            want, exponents = ref.quantize_weight(part, fmt)
            assert torch.equal(ref.decode(c[e], fmt), want) and torch.equal(s[e].long(), exponents + 127)
    alone = sb.quantize_weight_f8_block(given.to(DEV), fmt, transpose=False)
    assert torch.equal(alone[0].cpu(), out[0]) and torch.equal(alone[1].cpu(), out[1]) and alone[2] is None and alone[3] is None


def random_offsets(b, experts, gen, first=0, rest=0):
    """Ragged, with empty experts at both ends and in between."""
    cuts = torch.randint(first, b - rest + 1, (experts - 1,), generator=gen).sort().values.tolist()
    at = [first] + cuts + [b - rest]
    if experts >= 4:
        at[1] = at[0]
        at[-2] = at[-1]
        at[experts // 2] = at[experts // 2 + 1]
    return sorted(at)


#: M, N, K, experts (0: plain), rows before the first and behind the last one's
PRODUCTS = [(1, 64, 128, 0, 0, 0), (31, 192, 384, 0, 0, 0), (65, 64, 640, 0, 0, 0), (300, 256, 1152, 0, 0, 0), (513, 320, 128, 0, 0, 0),
            (1100, 576, 256, 0, 0, 0), (2500, 1088, 512, 0, 0, 0), (700, 4160, 384, 0, 0, 0), (1, 128, 128, 3, 0, 0), (5, 64, 256, 8, 0, 0), (40, 192, 384, 4, 1, 2),
            (333, 128, 640, 5, 0, 0), (1000, 320, 128, 7, 3, 57), (900, 1088, 512, 2, 0, 0), (1500, 640, 256, 33, 0, 100),
            (64, 64, 1152, 100, 0, 0), (3000, 576, 384, 6, 0, 11), (200, 64, 128, 1024, 0, 0), (5000, 2624, 256, 9, 0, 0),
            # plain: whole 256x256 tiles and the last rows apart; tiles of both kinds; 256x128; 256x256; 64x64 blocks of two waves
            (16406, 832, 256, 0, 0, 0), (16665, 960, 640, 0, 0, 0), (644, 3008, 128, 0, 0, 0), (1003, 4096, 1152, 0, 0, 0), (16406, 448, 128, 0, 0, 0),
            (4011, 2880, 1152, 0, 0, 0), (200, 2368, 128, 0, 0, 0),
            # by experts: 64x64 blocks of four and of two waves, 256x128 and 256x256 tiles, more than 64 experts on tiles
            (30, 1152, 512, 47, 0, 0), (30, 576, 128, 47, 0, 0), (372, 2752, 128, 11, 0, 0), (2011, 2048, 2048, 8, 0, 0), (5003, 1088, 768, 24, 5, 61),
            (9000, 1152, 256, 150, 1, 70)]


@pytest.mark.parametrize("M,N,K,experts,first,rest", PRODUCTS)
def test_products_are_exact_where_nothing_is_dropped(M, N, K, experts, first, rest):
    """Codes 0, 1/4, 1/2, 1 and scales that differ in every block: every sum is exact in binary32, so that a wrong scale, row,
    column, block or expert shows.  Rows of no expert keep what they held."""
    gen = torch.Generator().manual_seed(M + N + K + experts)
    pick = lambda *s: torch.tensor([0.0, 0.25, 0.5, 1.0])[torch.randint(0, 4, s, generator=gen)] * (torch.randint(0, 2, s, generator=gen) * 2 - 1)
    kb, nb, E = K // 128, -(-N // 128), experts or 1
    a, b = pick(M, K).double(), pick(E, N, K).double()
    ea, eb = torch.randint(-2, 3, (M, kb), generator=gen), torch.randint(-2, 3, (E, nb, kb), generator=gen)
    offsets = random_offsets(M, experts, gen, first, rest) if experts else None
    scales_a = row_scales(ea)
    weights = torch.stack([ref.weight_values(b[e], eb[e]) for e in range(E)])
    want, _ = ref.product(ref.row_values(a, ea), weights if experts else weights[0], offsets, untouched=-7.0)
    on = lambda t: (t if experts else t[0]).contiguous().to(DEV)
    where = torch.tensor(offsets, dtype=torch.int32, device=DEV) if experts else None
    for fmt_a, fmt_b in ((E4M3, E4M3), (E5M2, E4M3), (E4M3, E5M2), (E5M2, E5M2)):
        for dtype in (torch.float32, torch.bfloat16):
            out = torch.full((M, N), -7.0, dtype=dtype, device=DEV)
            sb.matmul_f8_block(ref.encode(a, fmt_a).to(DEV), fmt_a, scales_a.to(DEV), on(ref.encode(b, fmt_b)), fmt_b,
                               on((eb + 127).to(torch.uint8)), offsets=where, out=out)
            assert torch.equal(out.cpu(), want.to(dtype)), (fmt_a, fmt_b, dtype)


def test_scales_at_both_ends():
    """The lowest and the highest scale bytes there are, and products of them that binary32 still holds."""
    K = 256
    a, b = torch.ones(3, K), torch.ones(64, K)
    ea = torch.tensor([[-127, -127], [120, -127], [-60, 120]])
    eb = torch.tensor([[0, 120]])
    scales_a = row_scales(ea)
    want, _ = ref.product(ref.row_values(a.double(), ea), ref.weight_values(b.double(), eb))
    out = sb.matmul_f8_block(ref.encode(a, 0).to(DEV), 0, scales_a.to(DEV), ref.encode(b, 0).to(DEV), 0,
                             (eb + 127).to(torch.uint8).to(DEV), out_dtype=torch.float32)
    finite = want.abs() < 3e38
    assert torch.equal(out.cpu()[finite].double(), want[finite].float().double()) and torch.isinf(out.cpu()[~finite]).all()


#: b, n, m, experts, rows behind the last one's
LAYERS = [(1, 64, 64, None, 0), (37, 192, 320, None, 0), (512, 256, 1024, None, 0), (1029, 1088, 576, None, 0), (2000, 640, 2624, None, 0),
          (9, 64, 192, 4, 2), (700, 320, 192, 5, 0), (1500, 576, 1088, 12, 31), (48, 256, 512, 32, 0), (3000, 448, 1280, 3, 0)]


def layer(b, n, m, experts, rest, seed=0):
    gen = torch.Generator().manual_seed(seed + b + n + m)
    x = torch.randn(b, n, generator=gen)
    x[:, ::97] *= 50.0
    dy = 0.1 * torch.randn(b, m, generator=gen)
    w = torch.randn(experts or 1, m, n, generator=gen) / n ** 0.5
    offsets = random_offsets(b, experts, gen, 0, rest) if experts else None
    return x.bfloat16(), dy.bfloat16(), w.bfloat16(), offsets


@pytest.mark.parametrize("b,n,m,experts,rest", LAYERS)
def test_layer(b, n, m, experts, rest):
    """Forward, input gradient and weight gradient, and serving on the kept codes."""
    x, dy, w, offsets = layer(b, n, m, experts, rest)
    wd = (w if experts else w[0]).contiguous().to(DEV)
    where = torch.tensor(offsets, dtype=torch.int32, device=DEV) if experts else None
    values = torch.stack([ref.weight_values(*ref.quantize_weight(part, E4M3))[:, :n] for part in w])
    xv, gv = ref.row_values(*ref.quantize_rows(x, E4M3))[:, :n], ref.row_values(*ref.quantize_rows(dy, E5M2))[:, :m]
    want, size = ref.product(xv, values if experts else values[0], offsets)
    want_dx, size_dx = ref.product(gv, values.transpose(1, 2) if experts else values[0].t(), offsets)
    bufs = sb.BlockBuffers(b, n, m, experts)
    for dtype in (torch.bfloat16, torch.float32):
        y, dx = torch.zeros(b, m, dtype=dtype, device=DEV), torch.zeros(b, n, dtype=dtype, device=DEV)
        sb.forward_f8_block(x.to(DEV), wd, bufs, offsets=where, y=y)
        sb.backward_input_f8_block(dy.to(DEV), bufs, offsets=where, dx=dx)
        within(y, want, product_tol(size, n), "y")
        within(dx, want_dx, product_tol(size_dx, m), "dx")
        kept = torch.zeros_like(y)
        sb.linear_f8_block(x.to(DEV), bufs.wq, bufs.scales_w, offsets=where, y=kept)
        within(kept, want, product_tol(size, n), "y on kept codes")
        dw = (sb.backward_weight_experts(dy.to(DEV), x.to(DEV), where, bufs, dw_dtype=dtype) if experts else
              sb.backward_weight(dy.to(DEV), x.to(DEV), bufs, dw_dtype=dtype)[None])
        for e, rows in enumerate(ref.expert_slices(offsets or [0, b], b)):
            g, v = dy[rows].double().t(), x[rows].double()
            within(dw[e], g @ v, (b / 32 + 64) * 2.0 ** -23 * (g.abs() @ v.abs()), "dw")


@pytest.mark.parametrize("b,n,m,experts,rest", [(1, 64, 64, None, 0), (1, 4096, 192, None, 0), (16, 576, 320, None, 0), (17, 576, 320, None, 0), (7, 1088, 64, None, 0),
                                                (5, 128, 64, 8, 1), (60, 320, 128, 16, 3), (96, 2048, 96 * 2, 24, 0), (64, 192, 64, 16, 0),
                                                (100, 1024, 256, None, 0), (500, 576, 192, None, 0), (333, 320, 256, 5, 7), (1000, 128, 64, 3, 0)])
@FMT
def test_serving_a_few_rows(b, n, m, experts, rest, fmt):
    """Rows that the product quantizes itself: codes and scales as those of the quantizer, so that products which lose nothing
    are equal; rows with zeros, ties, subnormals and the largest values; all rows of 16 experts on one of them."""
    x, _, w, offsets = layer(b, n, m, experts, rest)
    edge_rows(x)
    gen = torch.Generator().manual_seed(4)
    if experts == 16 and rest == 0:
        offsets = [0] * 8 + [b] * 9
    where = torch.tensor(offsets, dtype=torch.int32, device=DEV) if experts else None
    coded = [ref.quantize_weight(part, E4M3) for part in w]
    stack = lambda ts: (torch.stack(ts) if experts else ts[0]).contiguous().to(DEV)
    codes, scales = stack([ref.encode(c, E4M3) for c, _ in coded]), stack([(e + 127).to(torch.uint8) for _, e in coded])
    values = torch.stack([ref.weight_values(c, e)[:, :n] for c, e in coded])
    xv = ref.row_values(*ref.quantize_rows(x, fmt))[:, :n]
    want, size = ref.product(xv, values if experts else values[0], offsets, untouched=3.0)
    for dtype in (torch.float32, torch.bfloat16):
        y = torch.full((b, m), 3.0, dtype=dtype, device=DEV)
        sb.linear_f8_block(x.to(DEV), codes, scales, offsets=where, fmt_x=fmt, y=y)
        fits = size < 1e38  # of the row with the largest value
        within(y.cpu()[fits], want[fits], product_tol(size[fits], n), "y")
    # One value a block, the others zero: nothing is dropped, every sum is exact.
    x = torch.zeros(b, n)
    for i in range(b):
        for k in range(0, n, 128):
            x[i, k + int(torch.randint(0, min(128, n - k), (1,), generator=gen))] = (-1.0) ** i * 2.0 ** int(torch.randint(-8, 8, (1,), generator=gen))
    ones = torch.ones(experts or 1, m, -(-n // 128) * 128)
    w_codes = ref.encode(ones, E4M3).to(DEV)
    exact, _ = ref.product(x.double(), torch.ones(experts, m, n, dtype=torch.float64) if experts else torch.ones(m, n, dtype=torch.float64), offsets)
    y = torch.zeros(b, m, device=DEV)
    sb.linear_f8_block(x.bfloat16().to(DEV), w_codes if experts else w_codes[0], torch.full_like(scales, 127), offsets=where, fmt_x=fmt, y=y)
    assert torch.equal(y.cpu(), exact.float())


@pytest.mark.parametrize("b,n,m,experts", [(1, 64, 64, 1), (3, 64, 128, 3), (1000, 128, 64, 2), (5000, 320, 192, 3), (3001, 1088, 576, 9),
                                           (777, 256, 320, 40), (20000, 256, 256, 2), (4100, 1280, 768, 5), (0, 64, 192, 4), (12000, 64, 1216, 6),
                                           (300, 1088, 1216, 24), (2500, 1344, 1344, 12), (40, 704, 960, 64)])
def test_weight_gradient_of_experts(b, n, m, experts):
    """Small tiles and large ones, split sums and whole ones, experts without rows, rows of no expert (which may hold NaN)."""
    gen = torch.Generator().manual_seed(b + n)
    x, dy = torch.randn(b, n, generator=gen).bfloat16(), torch.randn(b, m, generator=gen).bfloat16()
    rest = min(b // 10, 33)
    offsets = random_offsets(b, experts, gen, 0, rest)
    if rest:
        x[b - rest:], dy[b - rest:] = float("nan"), float("inf")
    where = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    for dtype in (torch.float32, torch.bfloat16):
        out = [sb.backward_weight_experts(dy.to(DEV), x.to(DEV), where, dw_dtype=dtype) for _ in range(2)]
        assert torch.equal(*out)
        for e, rows in enumerate(ref.expert_slices(offsets, b)):
            g, v = dy[rows].double().t(), x[rows].double()
            within(out[0][e], g @ v, (b / 32 + 64) * 2.0 ** -23 * (g.abs() @ v.abs()), "dw of expert %d" % e)


def test_offsets_out_of_range_stay_within_the_rows():
    """What the documentation leaves unspecified: offsets past b, below zero and decreasing are clamped."""
    x, dy, w, _ = layer(130, 64, 128, 3, 0)
    bufs = sb.BlockBuffers(130, 64, 128, 3)
    for offsets in ([0, 50, 130, 4000], [-7, 20, 90, 130], [0, 90, 40, 130], [200, 300, 400, 500], [0, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 5, 9]):
        where = torch.tensor(offsets, dtype=torch.int32, device=DEV)
        y, _ = sb.forward_f8_block(x.to(DEV), w.to(DEV), bufs, offsets=where)
        sb.backward_input_f8_block(dy.to(DEV), bufs, offsets=where)
        sb.backward_weight_experts(dy.to(DEV), x.to(DEV), where, bufs)
        torch.cuda.synchronize()
    # The clamped ones are those that they are clamped to.
    ys = [sb.forward_f8_block(x.to(DEV), w.to(DEV), bufs, offsets=torch.tensor(o, dtype=torch.int32, device=DEV))[0]
          for o in ([-7, 50, 130, 4000], [0, 50, 130, 130])]
    assert torch.equal(*ys)


def test_no_rows():
    x = torch.empty(0, 128, dtype=torch.bfloat16, device=DEV)
    w = torch.randn(64, 128, device=DEV).bfloat16()
    y, bufs = sb.forward_f8_block(x, w)
    codes = sb.quantize_weight_f8_block(w, E4M3)
    assert y.shape == (0, 64) and torch.equal(bufs.wq, codes[0]) and torch.equal(bufs.scales_wt, codes[3])
    assert sb.linear_f8_block(x, bufs.wq, bufs.scales_w).shape == (0, 64)
    assert sb.quantize_rowwise_f8_block(x, E4M3)[0].shape == (0, 128)
    assert sb.backward_input_f8_block(torch.empty(0, 64, dtype=torch.bfloat16, device=DEV), bufs).shape == (0, 128)


def test_gradients_against_differences():
    """The layer's gradients are those of the product of what the codes stand for, which is linear: differences in 64 bits of a
    loss along random directions."""
    b, n, m, experts = 90, 128, 64, 3
    x, dy, w, offsets = layer(b, n, m, experts, 4)
    where = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    bufs = sb.BlockBuffers(b, n, m, experts)
    sb.forward_f8_block(x.to(DEV), w.to(DEV), bufs, offsets=where)
    dx = torch.zeros(b, n, device=DEV)
    sb.backward_input_f8_block(dy.to(DEV), bufs, offsets=where, dx=dx)
    dw = sb.backward_weight_experts(dy.to(DEV), x.to(DEV), where, bufs, dw_dtype=torch.float32)
    values = torch.stack([ref.weight_values(*ref.quantize_weight(part, E4M3))[:, :n] for part in w])
    g = ref.row_values(*ref.quantize_rows(dy, E5M2))[:, :m]
    gen = torch.Generator().manual_seed(1)
    along = torch.randn(b, n, generator=gen, dtype=torch.float64)
    slope = sum((ref.product(x.double() + s * along, values, offsets)[0] * g).sum() / (2 * s) for s in (0.5, -0.5))
    assert abs(float((dx.cpu().double() * along).sum() - slope)) <= float((product_tol(ref.product(g, values.transpose(1, 2), offsets)[1], m) * along.abs()).sum())
    along = torch.randn(w.shape, generator=gen, dtype=torch.float64)
    slope = sum((ref.product(x.double(), w.double() + s * along, offsets)[0] * dy.double()).sum() / (2 * s) for s in (0.5, -0.5))
    size = torch.stack([dy[r].double().abs().t() @ x[r].double().abs() for r in ref.expert_slices(offsets, b)])
    assert abs(float((dw.cpu().double() * along).sum() - slope)) <= float((size * along.abs()).sum()) * (b / 32 + 64) * 2.0 ** -23


def block_step(x, dy, gamma, beta, w, where, bufs, keep):
    """A pre-norm layer of experts: norm, layer, gradients back through both."""
    sb.layer_norm(x, gamma, beta, y=keep["h"], mean=keep["mean"], rstd=keep["rstd"])
    sb.forward_f8_block(keep["h"], w, bufs, offsets=where, y=keep["y"])
    sb.backward_input_f8_block(dy, bufs, offsets=where, dx=keep["dh"])
    sb.backward_weight_experts(dy, keep["h"], where, bufs, dw=keep["dw"])
    sb.layer_norm_backward(keep["dh"], x, keep["mean"], keep["rstd"], gamma, dx=keep["dx"], dgamma=keep["dgamma"], dbeta=keep["dbeta"], ws=keep["ws"])


def kept(b, n, m, experts):
    e = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device=DEV)
    f = lambda *s: e(*s, dtype=torch.float32)
    return {"h": e(b, n), "mean": f(b), "rstd": f(b), "y": e(b, m), "dh": e(b, n), "dw": f(experts, m, n), "dx": e(b, n), "dgamma": f(n),
            "dbeta": f(n), "ws": torch.empty(sb.workspace_bytes(sb.SB_OP_LAYER_NORM_BACKWARD, b, n, 0), dtype=torch.uint8, device=DEV)}


def test_norm_and_experts_together():
    """Each result against the 64-bit form on the GPU's own results before it."""
    b, n, m, experts = 1111, 320, 448, 6
    x, dy, w, offsets = layer(b, n, m, experts, 20)
    gen = torch.Generator().manual_seed(2)
    gamma, beta = 1.0 + 0.2 * torch.randn(n, generator=gen), 0.1 * torch.randn(n, generator=gen)
    keep = kept(b, n, m, experts)
    where = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    block_step(x.to(DEV), dy.to(DEV), gamma.to(DEV), beta.to(DEV), w.to(DEV), where, sb.BlockBuffers(b, n, m, experts), keep)
    k = {name: t.cpu() for name, t in keep.items()}
    h, _, _ = ref.layer_norm(x, gamma, beta, 1e-5)
    within(keep["h"], h, 2.0 ** -15 * (1 + h.abs()), "norm")
    values = torch.stack([ref.weight_values(*ref.quantize_weight(part, E4M3))[:, :n] for part in w])
    y, size = ref.product(ref.row_values(*ref.quantize_rows(k["h"], E4M3))[:, :n], values, offsets)
    within(keep["y"], y, product_tol(size, n), "y")
    dh, size = ref.product(ref.row_values(*ref.quantize_rows(dy, E5M2))[:, :m], values.transpose(1, 2), offsets)
    within(keep["dh"], dh, product_tol(size, m), "dh")
    for e, rows in enumerate(ref.expert_slices(offsets, b)):
        g, v = dy[rows].double().t(), k["h"][rows].double()
        within(keep["dw"][e], g @ v, (b / 32 + 64) * 2.0 ** -23 * (g.abs() @ v.abs()), "dw")
    dx, dg, db, hh, a = ref.layer_norm_backward(k["dh"], x, k["mean"], k["rstd"], gamma)
    r = k["rstd"].double()[:, None]
    within(keep["dx"], dx, 2.0 ** -17 * r * (a.abs() + a.abs().mean(1, keepdim=True) + 2 * hh.abs() * (a * hh).abs().mean(1, keepdim=True)), "dx")
    within(keep["dgamma"], dg, 2.0 ** -16 * (k["dh"].double() * hh).abs().sum(0), "dgamma")
    within(keep["dbeta"], db, 2.0 ** -16 * k["dh"].double().abs().sum(0), "dbeta")


def test_captured_in_graphs_and_on_two_streams():
    """Two captured steps with buffers of their own, replayed with other inputs and other offsets, one after the other and side by
    side: the eager results every time."""
    b, n, m, experts = 700, 192, 320, 4
    sides = []
    for seed in (0, 1):
        x, dy, w, offsets = layer(b, n, m, experts, 10, seed)
        t = {"x": x.to(DEV), "dy": dy.to(DEV), "w": w.to(DEV), "where": torch.tensor(offsets, dtype=torch.int32, device=DEV),
             "gamma": torch.rand(n, device=DEV), "beta": torch.rand(n, device=DEV), "bufs": sb.BlockBuffers(b, n, m, experts), "keep": kept(b, n, m, experts),
             "stream": torch.cuda.Stream(), "graph": torch.cuda.CUDAGraph()}
        step = lambda t=t: block_step(t["x"], t["dy"], t["gamma"], t["beta"], t["w"], t["where"], t["bufs"], t["keep"])
        torch.cuda.synchronize()
        with torch.cuda.stream(t["stream"]):
            step()
        torch.cuda.synchronize()
        with torch.cuda.graph(t["graph"], stream=t["stream"]):
            step()
        t["step"] = step
        sides.append(t)
    gen = torch.Generator().manual_seed(9)
    for i in range(3):
        for t in sides:
            t["x"].copy_(torch.randn(b, n, generator=gen).bfloat16())
            t["dy"].copy_(torch.randn(b, m, generator=gen).bfloat16())
            t["where"].copy_(torch.tensor(random_offsets(b, experts, gen, 0, 5 * i), dtype=torch.int32))
            for name in ("y", "dh"):
                t["keep"][name].zero_()
        torch.cuda.synchronize()
        for t in sides:
            with torch.cuda.stream(t["stream"]):
                t["graph"].replay()
        torch.cuda.synchronize()
        for t in sides:
            replayed = {name: v.clone() for name, v in t["keep"].items() if name != "ws"}
            for name in ("y", "dh"):
                t["keep"][name].zero_()
            t["step"]()
            torch.cuda.synchronize()
            assert all(torch.equal(v, t["keep"][name]) for name, v in replayed.items()), "replay %d" % i


def test_memory_that_no_kernel_may_touch_is_refused():
    """Workspaces and buffers on the host, outputs over inputs."""
    x, dy, w = (torch.randn(600, 1024, device=DEV).bfloat16(), torch.randn(600, 1024, device=DEV).bfloat16(), torch.randn(1024, 1024, device=DEV).bfloat16())
    y, bufs = sb.forward_f8_block(x, w)
    need = sb.load_library().switchback_linear_f8_block_workspace_bytes(600, 1024, 1024, 1)
    assert need > 0
    with pytest.raises(sb.SwitchBackError):
        sb.linear_f8_block(x, bufs.wq, bufs.scales_w, ws=torch.zeros(need, dtype=torch.uint8))
    with pytest.raises(sb.SwitchBackError):
        sb.forward_f8_block(x, w, sb.BlockBuffers(600, 1024, 1024, None, "cpu"))
    with pytest.raises(sb.SwitchBackError):
        sb.backward_input_f8_block(dy, sb.BlockBuffers(600, 1024, 1024, None, "cpu"))
    with pytest.raises(sb.SwitchBackError):
        sb.backward_weight_experts(dy, x, torch.tensor([0, 600], dtype=torch.int32, device=DEV), sb.BlockBuffers(600, 1024, 1024, 1, "cpu"))
    for rows in (600, 4):
        with pytest.raises(sb.SwitchBackError):
            sb.backward_input_f8_block(dy[:rows], sb.BlockBuffers(rows, 1024, 1024), dx=dy[:rows])
        with pytest.raises(sb.SwitchBackError):
            sb.linear_f8_block(x[:rows], bufs.wq, bufs.scales_w, y=x[:rows])
    ws = torch.zeros(need, dtype=torch.uint8, device=DEV)
    assert torch.equal(sb.linear_f8_block(x, bufs.wq, bufs.scales_w, ws=ws), y)
    with pytest.raises(sb.SwitchBackError):
        sb.layer_norm(x, y=x)


def test_serving_captured_in_a_graph():
    """The few-rows kernel, replayed with other rows and offsets."""
    b, n, m, experts = 13, 320, 192, 5
    gen = torch.Generator().manual_seed(4)
    w = torch.randn(experts, m, n, generator=gen).bfloat16().to(DEV)
    codes, scales, _, _ = sb.quantize_weight_f8_block(w, E4M3)
    x, y = torch.zeros(b, n, dtype=torch.bfloat16, device=DEV), torch.zeros(b, m, dtype=torch.bfloat16, device=DEV)
    where = torch.zeros(experts + 1, dtype=torch.int32, device=DEV)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        sb.linear_f8_block(x, codes, scales, offsets=where, y=y)
    for i in range(4):
        x.copy_(torch.randn(b, n, generator=gen).bfloat16())
        where.copy_(torch.tensor(random_offsets(b, experts, gen, 0, i), dtype=torch.int32))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = sb.linear_f8_block(x, codes, scales, offsets=where, y=torch.zeros_like(y))
        assert torch.equal(y, eager), "replay %d" % i


def test_experts_behind_four_gib():
    """Weights, codes and gradients of the last experts lie behind 2^32 bytes: each expert's results are those of its own weight."""
    experts, m, n = 5, 16384, 16384
    # Values of one binary digit, and scales of one: nothing is dropped, and sums of up to 2^15 of them are exact.
    gen = torch.Generator(device=DEV).manual_seed(1)
    w = torch.empty(experts, m, n, dtype=torch.bfloat16, device=DEV)
    for e in range(experts):
        w[e] = torch.randint(-1, 2, (m, n), generator=gen, device=DEV, dtype=torch.int8)
    codes, scales, codes_t, scales_t = sb.quantize_weight_f8_block(w, E4M3)
    for e in (0, experts - 1):
        alone = sb.quantize_weight_f8_block(w[e], E4M3)
        assert all(torch.equal(t[e], one) for t, one in zip((codes, scales, codes_t, scales_t), alone))
    for counts in ([3, 0, 0, 2, 4], [100, 20, 0, 60, 300]):
        b = sum(counts)
        where = torch.tensor([sum(counts[:e]) for e in range(experts + 1)], dtype=torch.int32, device=DEV)
        x = torch.randint(-1, 2, (b, n), generator=gen, device=DEV, dtype=torch.int8).bfloat16()
        y = sb.linear_f8_block(x, codes, scales, offsets=where, y_dtype=torch.float32)
        dx = sb.linear_f8_block(x, codes_t, scales_t, offsets=where, y_dtype=torch.float32)
        dw = sb.backward_weight_experts(x, x, where, dw_dtype=torch.float32)
        for e in range(experts):
            rows = slice(int(where[e]), int(where[e + 1]))
            for got, weight in ((y, w[e]), (dx, w[e].t().contiguous())):
                assert torch.equal(got[rows], x[rows].float() @ weight.float().t()), "expert %d of %s" % (e, counts)
            assert torch.equal(dw[e, -512:], x[rows, -512:].float().t() @ x[rows].float()), "gradient of expert %d of %s" % (e, counts)


@pytest.mark.parametrize("counts", [[4971, 2444, 2452, 4249, 0, 0, 2332, 0], [2056] * 8, [16384, 0, 0, 0, 0, 0, 0, 64], [64, 16384, 0, 0, 0, 0, 0, 0],
                                    [300] * 7 + [14348], [16448, 0, 0, 0, 0, 0, 0, 0], [100] * 7 + [15000]],
                         ids=["uneven", "even", "whole", "first", "last", "one", "padded"])
def test_last_tile_rows_of_experts(counts):
    """A contraction of 4096 for 16448 rows of 8 experts: where the last round of tiles is nearly empty, its rows are the
    small-product kernel's.  Values of one binary digit: every sum is exact."""
    b, n, m, experts = 16448, 4096, 1024, 8
    gen = torch.Generator(device=DEV).manual_seed(3)
    w = torch.randint(-1, 2, (experts, m, n), generator=gen, device=DEV, dtype=torch.int8).bfloat16()
    x = torch.randint(-1, 2, (b, n), generator=gen, device=DEV, dtype=torch.int8).bfloat16()
    where = torch.tensor([sum(counts[:e]) for e in range(experts + 1)], dtype=torch.int32, device=DEV)
    codes, scales, _, _ = sb.quantize_weight_f8_block(w, E4M3)
    for dtype in (torch.bfloat16, torch.float32):
        y = torch.full((b, m), -7.0, dtype=dtype, device=DEV)
        sb.linear_f8_block(x, codes, scales, offsets=where, y=y)
        for e in range(experts):
            rows = slice(int(where[e]), int(where[e + 1]))
            assert torch.equal(y[rows], (x[rows].float() @ w[e].float().t()).to(dtype)), "expert %d" % e
        assert (y[sum(counts):] == -7.0).all()
