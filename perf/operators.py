"""The operators around the 8-bit linear layers, as a set of measured cases over the public Python entry points.

A case is a dict of plain values.  "kind" names the operator and its direction:

  norm_forward    layer norm of b rows of n columns: rows, means, reciprocal standard deviations
  norm_backward   its gradients: of the rows, of the weight and of the bias (sums over all rows)
  block_forward   the float8 layer n -> m with a scale for each block of 128: X and W quantized, the product
  block_step      a training step of it: forward, input gradient (dY in E5M2), 16-bit weight gradient
  block_serve     serving: rows quantized, product with weight codes that were laid out once
  expert_step     a training step with a weight per expert, rows sorted by expert, ragged counts
  expert_serve    serving with a weight per expert

b is the number of rows (tokens), "type" that of the layer norm's rows, "dw" that of the weight gradient, "data" the
distribution of X and dY ("outlier": 0.1 % of X's feature columns a hundred times larger, dY heavy-tailed).  "experts",
"spread", "rest" and "routing" say how the rows fall on experts: how uneven, how many at the end belong to none, and which
routing of these it is.

Block scales are powers of two, 2^e with the least e >= -127 for which the block's largest magnitude is at most the format's
largest value times 2^e; rows have blocks of 1 x 128, weights of 128 x 128.
"""
import math
import random

import torch

own = False

EPS = 1e-5
E4M3, E5M2 = 0, 1  # as the package numbers the formats


def _norm(name, kind, b, n, type="bf16"):
    return {"name": name, "kind": kind, "b": b, "n": n, "type": type}


def _block(name, kind, b, n, m, dw="bf16", data="normal"):
    return {"name": name, "kind": kind, "b": b, "n": n, "m": m, "dw": dw, "data": data}


def _expert(name, kind, b, n, m, experts, spread, rest=0, routing=1, dw="bf16"):
    return {"name": name, "kind": kind, "b": b, "n": n, "m": m, "dw": dw, "data": "normal", "experts": experts,
            "spread": spread, "rest": rest, "routing": routing}


def listed():
    return [
        # The norm in front of a ViT-B/16 block while one 224-pixel image is served: a launch and its latency.
        _norm("image norm", "norm_forward", 197, 768),
        # The same in ViT-H/14 training with 128 images: nothing but memory traffic.
        _norm("vit_h14 norm", "norm_forward", 32896, 1280),
        # Gradients of a norm in binary32 with an odd number of packed tokens and a width that no power of two divides far.
        _norm("ragged norm backward f32", "norm_backward", 11237, 1088, type="f32"),
        # Gradients of the ViT-H/14 norm.
        _norm("vit_h14 norm backward", "norm_backward", 32896, 1280),
        # A unit-test sized layer: launches and host work.
        _block("tiny block step", "block_step", 512, 256, 1024),
        # Widths that are multiples of 64 but not of 128 (blocks cut short) and an odd number of tokens, binary32 gradient.
        _block("ragged block step", "block_step", 11237, 1088, 2880, dw="f32"),
        # ViT-H/14's first feed-forward layer in training.
        _block("vit_h14 fc1 block step", "block_step", 32896, 1280, 5120),
        # A large-language-model sized layer with outlier features, forward.
        _block("outlier up block forward", "block_forward", 16384, 4096, 16384, data="outlier"),
        # The same layer answering sixteen sequences, a token each: the weights' way from memory.
        _block("outlier up block serve", "block_serve", 16, 4096, 16384, data="outlier"),
        # Feed-forward experts on ViT-L/14 widths in training: eight experts, moderately uneven.
        _expert("vit_l14 experts step", "expert_step", 16448, 1024, 4096, 8, 0.3),
        # Many experts, some without a row, odd counts, a padded batch (the last rows belong to no expert).
        _expert("ragged experts step", "expert_step", 5003, 768, 1088, 24, 0.5, rest=61, dw="f32"),
        # Experts answering a few sequences: most experts have a row or two, the others none.
        _expert("experts serve", "expert_serve", 48, 1024, 4096, 32, 0.4),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["norm_forward", "norm_backward", "norm_backward", "block_forward", "block_step", "block_step",
                       "block_serve", "expert_step", "expert_step", "expert_serve"])
    if kind.startswith("norm"):
        while True:
            b, n = round(_log_uniform(rng, 1, 60000)), round(_log_uniform(rng, 64, 16384))
            if rng.random() < 0.6:  # most widths are multiples of 64
                n = max(64, n // 64 * 64)
            if b * n <= 32896 * 2560:
                return {"kind": kind, "b": b, "n": n, "type": rng.choice(["bf16", "bf16", "f32"])}
    serve = kind.endswith("serve")
    case = {"kind": kind, "b": 0, "n": 0, "m": 0, "dw": rng.choice(["bf16", "f32"]), "data": rng.choice(["normal", "normal", "outlier"])}
    while True:
        b = round(_log_uniform(rng, 1, 256) if serve else _log_uniform(rng, 16, 34000))
        n, m = (64 * max(1, round(_log_uniform(rng, 64, 8192) / 64)) for _ in range(2))
        experts = round(_log_uniform(rng, 2, 64)) if kind.startswith("expert") else 1
        if experts * n * m <= 1 << 27 and b * n * m <= 1 << 37 and b * max(n, m) <= 1 << 27:
            break
    case.update(b=b, n=n, m=m)
    if kind.startswith("expert"):
        case.update(data="normal", experts=experts, spread=round(rng.uniform(0.0, 0.6), 3), rest=rng.choice([0, 0, b // 50, b // 10]),
                    routing=rng.randrange(1 << 20))
    return case


# ---- What a user's program has in hand ---------------------------------------------------------------------------

def _counts(case):
    """Rows of every expert: one in eight experts has none, the others log-normal shares of the rows."""
    rng = random.Random(case["routing"])
    shares = [0.0 if rng.random() < 0.125 else math.exp(case["spread"] * rng.gauss(0.0, 1.0)) for _ in range(case["experts"])]
    if not any(shares):
        shares[0] = 1.0
    rows, total, seen, ends = case["b"] - case["rest"], sum(shares), 0.0, [0]
    for s in shares:
        seen += s
        ends.append(round(rows * seen / total))
    ends[-1] = rows
    return [end - begin for begin, end in zip(ends, ends[1:])]


def _activations(case, gen):
    b, n, m = case["b"], case["n"], case["m"]
    x = torch.randn(b, n, generator=gen, device="cuda")
    dy = torch.randn(b, m, generator=gen, device="cuda")
    if case["data"] == "outlier":
        x[:, torch.randperm(n, generator=gen, device="cuda")[: -(-n // 1000)]] *= 100.0
        chi2 = torch.randn(3, b, m, generator=gen, device="cuda").square_().sum(0)
        dy = dy.mul_(0.01).div_(chi2.div_(3.0).sqrt_())
    else:
        dy.mul_(0.1)
    return x.bfloat16(), dy.bfloat16()


def _offsets(case):
    return torch.tensor([0] + _counts(case), device="cuda").cumsum(0, dtype=torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    b, n = case["b"], case["n"]
    state = {"case": case}
    if case["kind"].startswith("norm"):
        # A residual stream: features of different magnitudes around means of their own.
        x = (normal(b, n) * (0.5 + normal(n).abs()) + 0.3 * normal(n)).to(torch.bfloat16 if case["type"] == "bf16" else torch.float32)
        state.update(x=x, gamma=1.0 + 0.2 * normal(n), beta=0.2 * normal(n))
        if case["kind"] == "norm_backward":
            wide = x.double()
            state.update(dy=(0.1 * normal(b, n)).to(x.dtype), mean=wide.mean(1).float(),
                         rstd=(1.0 / (wide.var(1, unbiased=False) + EPS).sqrt()).float())
        return state
    m, experts = case["m"], case.get("experts")
    x, dy = _activations(case, gen)
    shape = (m, n) if experts is None else (experts, m, n)
    w = (normal(*shape) / math.sqrt(n)).bfloat16()
    state.update(x=x, offsets=None, most=0)
    if experts is not None:
        state.update(offsets=_offsets(case), most=max(_counts(case)))
    if case["kind"].endswith("serve"):  # the weight's codes, laid out once
        codes, scales = _quantize_weight(w)
        state.update(codes=codes.to(torch.float8_e4m3fn).view(torch.uint8), scales=scales)
    else:
        state.update(w=w, dy=dy)
    # Outputs that the program keeps: rows of no expert stay as they were.
    state["y"] = torch.zeros(b, m, dtype=torch.bfloat16, device="cuda")
    if case["kind"].endswith("step"):
        state["dx"] = torch.zeros(b, n, dtype=torch.bfloat16, device="cuda")
    return state


# ---- The plain forms ---------------------------------------------------------------------------------------------

def _pad(t, dim, unit=128):
    """Zeros behind `dim` up to a multiple of `unit`."""
    more = -t.shape[dim] % unit
    if more == 0:
        return t
    shape = list(t.shape)
    shape[dim] = more
    return torch.cat([t, t.new_zeros(shape)], dim)


def _exponent(absmax, fmt):
    """Least e >= -127 with absmax <= MAX 2^e; MAX is 0.875 * 2^9 (E4M3) or 0.875 * 2^16 (E5M2)."""
    f, k = torch.frexp(absmax)
    e = k - (9 if fmt == E4M3 else 16) + (f > 0.875).int()
    return torch.where(absmax > 0, e, -127).clamp(min=-127)


def _times_power(x, e):
    """x * 2^e for -127 <= e <= 127; the power is made from its bits (2^-127 is subnormal), exactly."""
    return x * torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _to_f8(x, fmt):
    return x.to(torch.float8_e4m3fn if fmt == E4M3 else torch.float8_e5m2).float()


def _row_values(x, fmt):
    """What the row-wise codes of x [b, k] stand for, [b, k] in binary32."""
    blocks = _pad(x.float(), 1).view(x.shape[0], -1, 128)
    e = _exponent(blocks.abs().amax(2, keepdim=True), fmt)
    return _times_power(_to_f8(_times_power(blocks, -e), fmt), e).view(x.shape[0], -1)[:, :x.shape[1]]


def _quantize_weight(w):
    """Codes (as binary32 values, zeros behind the columns up to a multiple of 128) and scale bytes of w [.., m, n]."""
    m, n = w.shape[-2:]
    blocks = _pad(_pad(w.float(), -1), -2)
    rows, cols = blocks.shape[-2:]
    blocks = blocks.view(-1, rows // 128, 128, cols // 128, 128)
    e = _exponent(blocks.abs().amax((2, 4), keepdim=True), E4M3)
    codes = _to_f8(_times_power(blocks, -e), E4M3).view(*w.shape[:-2], rows, cols)[..., :m, :].contiguous()
    return codes, (e + 127).to(torch.uint8).view(*w.shape[:-2], rows // 128, cols // 128)


def _weight_values(codes, scales, n):
    """What codes with their scale bytes stand for."""
    m = codes.shape[-2]
    e = scales.int().sub(127).repeat_interleave(128, -2)[..., :m, :].repeat_interleave(128, -1)
    return _times_power(codes, e)[..., :n]


def _rows_of_experts(t, offsets, most):
    """t's rows by expert, [experts, most, ..], zeros behind the last one of each."""
    place = torch.arange(most, device=t.device)
    rows = (offsets[:-1, None] + place).clamp(max=t.shape[0] - 1)
    return t[rows] * (place < (offsets[1:] - offsets[:-1])[:, None])[..., None]


def _rows_in_place(t, offsets, b):
    """The reverse; rows of no expert are zeros."""
    rows = torch.arange(b, device=t.device)
    expert = torch.searchsorted(offsets[1:], rows, right=True)
    known = expert < t.shape[0]
    expert = expert.clamp(max=t.shape[0] - 1)
    return t.reshape(-1, t.shape[2])[(expert * t.shape[1] + rows - offsets[expert]).clamp(0, t.shape[0] * t.shape[1] - 1)] * known[:, None]


def _product(a, w, offsets, most):
    """a [b, k] times w [k, m], or by experts w [experts, k, m]."""
    if offsets is None:
        return a @ w
    return _rows_in_place(torch.bmm(_rows_of_experts(a, offsets, most), w.contiguous()), offsets, a.shape[0])


def _gradient_product(dy, x, offsets, most):
    if offsets is None:
        return dy.float().t() @ x.float()
    dy, x = (_rows_of_experts(t.float(), offsets, most) for t in (dy, x))
    return torch.bmm(dy.transpose(1, 2).contiguous(), x)


def _plain(state):
    case = state["case"]
    kind, n = case["kind"], case["n"]
    if kind == "norm_forward":
        x = state["x"].float()
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = 1.0 / ((x * x).mean(1) + EPS).sqrt()
        return {"y": (x * rstd[:, None] * state["gamma"] + state["beta"]).to(state["x"].dtype), "mean": mean, "rstd": rstd}
    if kind == "norm_backward":
        dy, rstd = state["dy"].float(), state["rstd"][:, None]
        h = (state["x"].float() - state["mean"][:, None]) * rstd
        a = dy * state["gamma"]
        dx = rstd * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
        return {"dx": dx.to(state["x"].dtype), "dgamma": (dy * h).sum(0), "dbeta": dy.sum(0)}
    offsets, most = state["offsets"], state["most"]
    if kind.endswith("serve"):
        w = _weight_values(state["codes"].view(torch.float8_e4m3fn).float(), state["scales"], n)
    else:
        w = _weight_values(*_quantize_weight(state["w"]), n)
    out = {"y": _product(_row_values(state["x"], E4M3), w.transpose(-1, -2), offsets, most).bfloat16()}
    if kind.endswith("step"):
        out["dx"] = _product(_row_values(state["dy"], E5M2), w, offsets, most).bfloat16()
        out["dw"] = _gradient_product(state["dy"], state["x"], offsets, most)
        out["dw"] = out["dw"].bfloat16() if case["dw"] == "bf16" else out["dw"]
    return out


def _own(state):
    from paper_2304_13013_amd import switchback as sb
    case = state["case"]
    kind = case["kind"]
    if kind == "norm_forward":
        y, mean, rstd = sb.layer_norm(state["x"], state["gamma"], state["beta"], eps=EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if kind == "norm_backward":
        dx, dgamma, dbeta = sb.layer_norm_backward(state["dy"], state["x"], state["mean"], state["rstd"], state["gamma"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    offsets = state["offsets"]
    if kind.endswith("serve"):
        return {"y": sb.linear_f8_block(state["x"], state["codes"], state["scales"], offsets=offsets, y=state["y"])}
    if "bufs" not in state:  # a layer's buffers, which a training program allocates once
        state["bufs"] = sb.BlockBuffers(case["b"], case["n"], case["m"], experts=case.get("experts"))
    bufs = state["bufs"]
    out = {"y": sb.forward_f8_block(state["x"], state["w"], bufs, offsets=offsets, y=state["y"])[0]}
    if kind.endswith("step"):
        dw_dtype = torch.bfloat16 if case["dw"] == "bf16" else torch.float32
        out["dx"] = sb.backward_input_f8_block(state["dy"], bufs, offsets=offsets, dx=state["dx"])
        if offsets is None:
            out["dw"] = sb.backward_weight(state["dy"], state["x"], bufs, dw_dtype=dw_dtype)
        else:
            out["dw"] = sb.backward_weight_experts(state["dy"], state["x"], offsets, bufs, dw_dtype=dw_dtype)
    return out


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    b, n, kind = case["b"], case["n"], case["kind"]
    if kind.startswith("norm"):
        size = 2 if case["type"] == "bf16" else 4
        if kind == "norm_forward":
            return {"bytes": 2 * b * n * size + 8 * b + 8 * n, "flops": 8 * b * n}
        return {"bytes": 3 * b * n * size + 8 * b + 12 * n, "flops": 14 * b * n}
    m, rows, experts = case["m"], b, 1
    if "experts" in case:
        rows, experts = b - case["rest"], sum(c > 0 for c in _counts(case))
    if kind.endswith("serve"):
        return {"bytes": 2 * rows * (n + m) + experts * n * m, "flops": 2 * rows * n * m}
    if kind == "block_forward":
        return {"bytes": 2 * (rows * n + n * m + rows * m), "flops": 2 * rows * n * m}
    every = case.get("experts", 1)  # the gradient of an expert without rows is written too
    return {"bytes": 4 * rows * (n + m) + 2 * experts * n * m + (2 if case["dw"] == "bf16" else 4) * every * n * m,
            "flops": 6 * rows * n * m}


# ---- The operators' definitions in 64 bits -------------------------------------------------------------------------

def _exact_power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_f8(v, digits, lowest):
    """v rounded to the nearest value with `digits` binary digits behind the first, of exponents from `lowest` on."""
    grid = _exact_power((torch.frexp(v)[1] - 1).clamp(min=lowest) - digits)
    return torch.round(v / grid) * grid


def _exact_codes(v, top, fmt):
    """v [.., block] scaled per block whose largest magnitude is `top`, rounded, and scaled back."""
    largest = 448.0 if fmt == E4M3 else 57344.0
    e = torch.frexp(top.clamp(min=2.0 ** -200) / largest)[1] - 2
    e = torch.where(top > largest * _exact_power(e), e + 1, e)
    e = torch.where(top > largest * _exact_power(e), e + 1, e)
    step = _exact_power(e.clamp(min=-127))
    return _exact_f8(v / step, *((3, -6) if fmt == E4M3 else (2, -14))) * step


def _exact_rows(x, fmt):
    return torch.cat([_exact_codes(part, part.abs().amax(1, keepdim=True), fmt) for part in x.double().split(128, 1)], 1)


def _exact_weight(w):
    return torch.cat([torch.cat([_exact_codes(part, part.abs().amax((-1, -2), keepdim=True), E4M3)
                                 for part in rows.split(128, -1)], -1) for rows in w.double().split(128, -2)], -2)


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("norm"):
        x, gamma = state["x"].double(), state["gamma"].double()
        if kind == "norm_forward":
            mean, spread = x.mean(1, keepdim=True), x.var(1, unbiased=False, keepdim=True)
            rstd = (spread + EPS).rsqrt()
            return {"y": (x - mean) * rstd * gamma + state["beta"].double(), "mean": mean[:, 0], "rstd": rstd[:, 0]}
        dy, mean, rstd = state["dy"].double(), state["mean"].double()[:, None], state["rstd"].double()[:, None]
        h, n = (x - mean) * rstd, case["n"]
        g = dy * gamma
        return {"dx": rstd / n * (n * g - g.sum(1, keepdim=True) - h * (g * h).sum(1, keepdim=True)),
                "dgamma": (dy * h).sum(0), "dbeta": dy.sum(0)}
    m, n = case["m"], case["n"]
    if kind.endswith("serve"):
        codes = state["codes"].view(torch.float8_e4m3fn).float().double()
        steps = _exact_power(state["scales"].int() - 127)
        w = torch.cat([torch.cat([part * steps[..., i:i + 1, j:j + 1] for j, part in enumerate(rows.split(128, -1))], -1)
                       for i, rows in enumerate(codes.split(128, -2))], -2)[..., :n]
    else:
        w = _exact_weight(state["w"])
    x, counts = _exact_rows(state["x"], E4M3), [case["b"]]
    if "experts" in case:
        counts = _counts(case)
    else:
        w = w[None]
    y = torch.zeros(case["b"], m, dtype=torch.float64, device="cuda")
    out = {"y": y}
    if kind.endswith("step"):
        dy, wide = _exact_rows(state["dy"], E5M2), state["x"].double()
        dx = torch.zeros(case["b"], n, dtype=torch.float64, device="cuda")
        dw = torch.zeros(len(counts), m, n, dtype=torch.float64, device="cuda")
        out.update(dx=dx, dw=dw if "experts" in case else dw[0])
    first = 0
    for e, count in enumerate(counts):
        rows = slice(first, first + count)
        first += count
        y[rows] = x[rows] @ w[e].t()
        if kind.endswith("step"):
            dx[rows] = dy[rows] @ w[e]
            dw[e] = state["dy"][rows].double().t() @ wide[rows]
    return out
