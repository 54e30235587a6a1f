"""The operators around the 8-bit layers in 64 bits, on the CPU, from their definitions: what the GPU tests compare with."""
import torch

E4M3, E5M2 = 0, 1
#: Largest value, binary digits behind the first, lowest exponent of a normal number.
FORMATS = {E4M3: (448.0, 3, -6), E5M2: (57344.0, 2, -14)}


def power(e):
    return torch.ldexp(torch.ones((), dtype=torch.float64), e)


def scale_exponent(absmax, fmt):
    """Least e >= -127 with absmax <= MAX 2^e, by trying: from below what it can be."""
    largest = FORMATS[fmt][0]
    e = torch.full(absmax.shape, -127, dtype=torch.int64)
    for _ in range(260):
        more = absmax > largest * power(e)
        if not more.any():
            break
        e += more
    return e


def to_format(v, fmt):
    """v rounded to nearest, ties to even, on the format's values."""
    _, digits, lowest = FORMATS[fmt]
    grid = power((torch.frexp(v)[1] - 1).clamp(min=lowest) - digits)
    return torch.round(v / grid) * grid


def quantize_rows(x, fmt):
    """(codes as values [rows, K], scale exponents [rows, K / 128]) of x [rows, cols]."""
    rows, cols = x.shape
    wide = torch.zeros(rows, -(-cols // 128) * 128, dtype=torch.float64)
    wide[:, :cols] = x.double()
    blocks = wide.view(rows, -1, 128)
    e = scale_exponent(blocks.abs().amax(2), fmt)
    return to_format(blocks / power(e)[:, :, None], fmt).view(rows, -1), e


def quantize_weight(w, fmt):
    """The same of w [m, n] in blocks of 128 x 128: (codes [m, K], exponents [blocks of m, K / 128])."""
    m, n = w.shape
    wide = torch.zeros(-(-m // 128) * 128, -(-n // 128) * 128, dtype=torch.float64)
    wide[:m, :n] = w.double()
    blocks = wide.view(wide.shape[0] // 128, 128, wide.shape[1] // 128, 128)
    e = scale_exponent(blocks.abs().amax((1, 3)), fmt)
    return to_format(blocks / power(e)[:, None, :, None], fmt).view(wide.shape)[:m], e


def row_values(codes, e):
    return (codes.view(e.shape[0], e.shape[1], 128) * power(e)[:, :, None]).view(codes.shape)


def weight_values(codes, e):
    return codes * power(e).repeat_interleave(128, 0)[:codes.shape[0]].repeat_interleave(128, 1)


def decode(codes, fmt):
    return codes.cpu().view(torch.float8_e4m3fn if fmt == E4M3 else torch.float8_e5m2).double()


def encode(values, fmt):
    return values.float().to(torch.float8_e4m3fn if fmt == E4M3 else torch.float8_e5m2).view(torch.uint8)


def expert_slices(offsets, b):
    at = [min(max(int(o), 0), b) for o in offsets]
    return [slice(first, end) for first, end in zip(at, at[1:])]


def product(a, w, offsets=None, untouched=0.0):
    """a [M, K] times w [N, K] (or the w of each row's expert) transposed, and the same of the magnitudes."""
    if offsets is None:
        return a @ w.t(), a.abs() @ w.abs().t()
    out = torch.full((a.shape[0], w.shape[1]), untouched, dtype=torch.float64)
    size = torch.zeros_like(out)
    for e, rows in enumerate(expert_slices(offsets, a.shape[0])):
        out[rows], size[rows] = a[rows] @ w[e].t(), a[rows].abs() @ w[e].abs().t()
    return out, size


def layer_norm(x, gamma, beta, eps):
    x = x.double()
    mean, var = x.mean(1), x.var(1, unbiased=False)
    rstd = 1.0 / torch.sqrt(var + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * gamma.double()
    if beta is not None:
        y = y + beta.double()
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, gamma):
    dy, r = dy.double(), rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r
    a = dy if gamma is None else dy * gamma.double()
    dx = r * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
    return dx, (dy * h).sum(0), dy.sum(0), h, a
