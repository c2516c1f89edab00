"""Cases for the operators around the attention of a layer: root-mean-square norm with the residual's addition, quantising to
8 bits, the product of 8-bit operands, and rotary positions.

8-bit operands are e4m3 codes with one power-of-two scale for each row and block of 128 columns: codes float8_e4m3fn
[rows, columns], scales float8_e8m0fnu [rows, 4 ceil(columns / 512)], whose entries behind the last block are one.  `run`
computes one pass in plain torch, or (with `own`) through the framework's calls.
"""
import math
import random

import torch

own = False

BLOCK, DIM = 128, 128
LOWEST = -126          # smallest exponent of a scale


# ------------------------------------------------------------------------------------------------ cases
def listed():
    def norm(name, rows, cols, residual, quantized):
        return dict(name=name, op="norm", rows=rows, cols=cols, residual=residual, quantized=quantized, eps=1e-5)

    def quantize(name, rows, cols):
        return dict(name=name, op="quantize", rows=rows, cols=cols)

    def product(name, rows, n, cols):
        return dict(name=name, op="product", rows=rows, n=n, cols=cols)

    def rotary(name, rows, hq, hkv, dim, layout, first, last, theta, scaling, factor, original):
        return dict(name=name, op="rotary", rows=rows, hq=hq, hkv=hkv, dim=dim, layout=layout, first=first, last=last,
                    theta=theta, scaling=scaling, factor=factor, original=original)

    return [
        # one user, one token: what counts is latency
        norm("norm answer", 1, 4096, True, True),
        # a long prompt, as operand of the projections behind it
        norm("norm prompt", 131072, 4096, True, True),
        # the last norm of a packed batch: no addition, 16 bits out
        norm("norm ragged", 9001, 3584, False, False),
        # the output of attention over a prompt, as operand of the projection behind it
        quantize("quantize context", 32768, 4096),
        # weights are laid out once, when a model is loaded
        quantize("quantize weight", 6144, 4096),
        # one token through the projection to Q, K and V of 32/8 heads
        product("product answer", 1, 6144, 4096),
        # a server's step through the projection behind attention
        product("product step", 33, 4096, 4096),
        # a follow-up question, 28/4 heads
        product("product piece", 700, 4608, 3584),
        # a prompt
        product("product prompt", 32768, 6144, 4096),
        # a server's step: every user at a position of its own
        rotary("rotary step", 32, 32, 8, 128, "half", 0, 131072, 500000.0, "bands", 8.0, 8192),
        # a long prompt
        rotary("rotary prompt", 131072, 32, 8, 128, "half", -1, 131072, 500000.0, "none", 1.0, 8192),
        # half of each head is rotated, in adjacent pairs
        rotary("rotary part", 5003, 28, 4, 64, "interleaved", 100, 40000, 10000.0, "linear", 4.0, 8192),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(("norm",) * 3 + ("quantize",) * 2 + ("product",) * 4 + ("rotary",) * 3)
    if op in ("norm", "quantize"):
        cols = 16 * _log(rng, 1, 1024)
        rows = _log(rng, 1, min(131072, (1 << 29) // cols))
        if op == "quantize":
            return dict(op=op, rows=rows, cols=cols)
        return dict(op=op, rows=rows, cols=cols, residual=rng.random() < 0.6, quantized=rng.random() < 0.6,
                    eps=rng.choice((1e-5, 1e-6)))
    if op == "product":
        cols, n = 16 * _log(rng, 4, 512), _log(rng, 16, 8192)
        most = 32768 * 6144 * 4096 // (n * cols)
        return dict(op=op, rows=_log(rng, 1, min(32768, most) if rng.random() < 0.5 else 256), n=n, cols=cols)
    hq, hkv = rng.choice(((4, 1), (32, 8), (28, 4), (8, 8), (16, 1), (6, 2)))
    rows, last = _log(rng, 1, 5242880 // (hq + 2 * hkv)), _log(rng, 64, 1 << 20)
    return dict(op=op, rows=min(rows, 131072), hq=hq, hkv=hkv, dim=16 * rng.randint(1, 8),
                layout=rng.choice(("half", "interleaved")), first=rng.choice((-1, 0, last // 2)), last=last,
                theta=rng.choice((10000.0, 500000.0, 1000000.0)), scaling=rng.choice(("none", "linear", "base", "ramp", "bands")),
                factor=rng.choice((2.0, 4.0, 8.0)), original=rng.choice((4096, 8192, 32768)))


def _words(cols):
    return -(-cols // 512)


def work(case):
    rows = case["rows"]
    if case["op"] == "rotary":
        return dict(bytes=rows * ((case["hq"] + 2 * case["hkv"]) * DIM * 4 + (4 if case["first"] >= 0 else 0)), flops=0)
    cols = case["cols"]
    codes = rows * (cols + 4 * _words(cols))
    if case["op"] == "quantize":
        return dict(bytes=rows * cols * 2 + codes, flops=0)
    if case["op"] == "norm":
        out = codes if case["quantized"] else rows * cols * 2
        return dict(bytes=rows * cols * (6 if case["residual"] else 2) + out + cols * 2, flops=0)
    return dict(bytes=codes + case["n"] * (cols + 4 * _words(cols)) + rows * case["n"] * 2, flops=2 * rows * case["n"] * cols)


# ------------------------------------------------------------------------------------------------ 8-bit operands
def _exponent(amax):
    """Smallest e >= LOWEST with amax <= 448 2^e, for finite amax >= 0 (exact; 448 is 1.75 2^8)."""
    m, k = torch.frexp(amax)
    e = torch.where(2 * m <= 1.75, k - 9, k - 8)
    return torch.where(amax > 0, e, torch.full_like(e, LOWEST)).clamp(min=LOWEST)


def _pow2(e):
    """2^e in float32 for integers -126 <= e <= 127 (the bits of the float)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _operand(y):
    """Codes and scales of float32 rows."""
    rows, cols = y.shape
    blocks = -(-cols // BLOCK)
    full = torch.nn.functional.pad(y, (0, blocks * BLOCK - cols)).view(rows, blocks, BLOCK)
    amax = torch.where(torch.isfinite(full), full.abs(), torch.zeros((), device=y.device)).amax(-1)
    e = _exponent(amax)
    codes = (full * _pow2(-e)[..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    scales = torch.full((rows, 4 * _words(cols)), 127, dtype=torch.uint8, device=y.device)
    scales[:, :blocks] = (e + 127).to(torch.uint8)
    return codes.view(rows, blocks * BLOCK)[:, :cols].contiguous(), scales.view(torch.float8_e8m0fnu)


def _value(codes, scales):
    """The float32 numbers that codes and scales stand for."""
    rows, cols = codes.shape
    blocks = -(-cols // BLOCK)
    s = (scales.view(torch.uint8)[:, :blocks].to(torch.int32) << 23).view(torch.float32)
    return codes.float() * s.repeat_interleave(BLOCK, 1)[:, :cols]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 17)
    rows, op = case["rows"], case["op"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.bfloat16)

    def states(n):
        """Hidden states: tokens of different size, a few strong channels."""
        x = normal(rows, n)
        x *= torch.rand(rows, 1, generator=gen, device=dev).mul_(1.5).add_(0.5).bfloat16()
        x[:, ::61] *= 12.0
        return x

    s = dict(case=case)
    if op == "norm":
        s["x"] = states(case["cols"])
        s["weight"] = (1.0 + 0.2 * normal(case["cols"]).float()).bfloat16()
        s["residual"] = states(case["cols"]).mul_(3.0) if case["residual"] else None
    elif op == "quantize":
        s["x"] = states(case["cols"])
    elif op == "product":
        s["codes"], s["scales"] = _operand(states(case["cols"]).float())
        s["w_codes"], s["w_scales"] = _operand(normal(case["n"], case["cols"]).float() * 0.02)
        if own:   # what a user's program keeps beside the weights
            import paper_2609_01925_b200 as crisp
            s["linear"] = crisp.CrispLinear(s["w_codes"], s["w_scales"])
    else:
        s["qkv"] = normal(rows, (case["hq"] + 2 * case["hkv"]) * DIM)
        s["positions"] = None   # the rows of one prompt, in order
        if case["first"] >= 0:
            s["positions"] = torch.randint(case["first"], case["last"], (rows,), generator=gen, device=dev).int()
        if own:
            import paper_2609_01925_b200 as crisp
            s["rotary"] = crisp.CrispRotary(case["theta"], rotary_dim=case["dim"], layout=case["layout"],
                                            scaling=case["scaling"], factor=case["factor"], original=case["original"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


def _own_norm(s):
    import paper_2609_01925_b200 as crisp
    call = crisp.rms_norm_quantize if s["case"]["quantized"] else crisp.rms_norm
    return call(s["x"], s["weight"], s["residual"], eps=s["case"]["eps"])


def _own_quantize(s):
    import paper_2609_01925_b200 as crisp
    return crisp.quantize(s["x"])


def _own_product(s):
    return s["linear"](s["codes"], s["scales"])


def _own_rotary(s):
    return s["rotary"].split(s["qkv"], s["case"]["hq"], s["case"]["hkv"], s["positions"])


def _plain_norm(s):
    x, total = s["x"], None
    if s["residual"] is not None:
        x = total = (x.float() + s["residual"].float()).bfloat16()
    h = x.float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + s["case"]["eps"]) * s["weight"].float()
    return (*_operand(y), total) if s["case"]["quantized"] else (y.bfloat16(), total)


def _plain_quantize(s):
    return _operand(s["x"].float())


def _plain_product(s):
    return (_value(s["codes"], s["scales"]) @ _value(s["w_codes"], s["w_scales"]).t()).bfloat16()


def _frequencies(case):
    """Angle per position of each pair, in float64 on the host, and the factor on what is rotated."""
    r, theta, factor, original = case["dim"], case["theta"], case["factor"], case["original"]
    f, size, kind = [], 1.0, case["scaling"]
    if kind == "base":
        theta *= factor ** (r / max(r - 2, 1))
    for i in range(r // 2):
        x = theta ** (-2 * i / r)
        if kind == "linear":
            x /= factor
        elif kind in ("ramp", "bands"):
            turns = original * x / (2 * math.pi)           # over the original length
            if kind == "bands":                            # 4 turns and more: kept; 1 and fewer: slowed
                keep = (turns - 1.0) / 3.0
            else:                                          # linear in i between the pairs with 32 turns and with 1
                at = [r * math.log(original / (2 * math.pi * t)) / (2 * math.log(theta)) for t in (32.0, 1.0)]
                lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
                keep = 1.0 - (i - lo) / max(hi - lo, 0.001)
            keep = min(max(keep, 0.0), 1.0)
            x = x * keep + x / factor * (1.0 - keep)
        f.append(x)
    if kind == "ramp":
        size = 0.1 * math.log(factor) + 1.0
    return f, size


def _plain_rotary(s):
    c = s["case"]
    rows, r, hq, hkv = c["rows"], c["dim"], c["hq"], c["hkv"]
    x = s["qkv"].view(rows, hq + 2 * hkv, DIM)
    f, size = _frequencies(c)
    pos = torch.arange(rows, device=x.device) if s["positions"] is None else s["positions"]
    angle = pos.double()[:, None] * torch.tensor(f, dtype=torch.float64).to(x.device)
    cos, sin = ((size * t).float()[:, None] for t in (angle.cos(), angle.sin()))

    def rotated(x):
        part = x[..., :r].float()
        if c["layout"] == "half":
            a, b = part[..., :r // 2], part[..., r // 2:]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = part[..., 0::2], part[..., 1::2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([turned.bfloat16(), x[..., r:]], -1)

    return rotated(x[:, :hq]), rotated(x[:, hq:hq + hkv]), x[:, hq + hkv:].contiguous()


_plain = dict(norm=_plain_norm, quantize=_plain_quantize, product=_plain_product, rotary=_plain_rotary)
_own = dict(norm=_own_norm, quantize=_own_quantize, product=_own_product, rotary=_own_rotary)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _e4m3_values(device):
    """The values of the e4m3 bytes 0 to 126, from the definition of the format."""
    out = []
    for c in range(127):
        e, m = c >> 3, c & 7
        out.append((1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6)
    return torch.tensor(out, dtype=torch.float64, device=device)


def _exact_operand(y):
    """Values of the nearest codes (ties to the even one) and of the scales, of float64 rows."""
    grid = _e4m3_values(y.device)
    rows, cols = y.shape
    values = torch.empty_like(y)
    scales = torch.ones(rows, 4 * _words(cols), dtype=torch.float64, device=y.device)
    for b in range(-(-cols // BLOCK)):
        part = y[:, b * BLOCK:(b + 1) * BLOCK]
        amax = part.abs().amax(1)
        e = torch.ceil(torch.log2(amax.clamp(min=1e-300) / 448))
        e = torch.where(amax > 448 * torch.exp2(e), e + 1, e)
        e = torch.where(amax <= 448 * torch.exp2(e - 1), e - 1, e).clamp(min=LOWEST)
        scales[:, b] = torch.exp2(e)
        a = (part.abs() / torch.exp2(e)[:, None]).clamp(max=448.0)
        hi = torch.searchsorted(grid, a).clamp(max=126)
        lo = (hi - 1).clamp(min=0)
        up, down = grid[hi] - a, a - grid[lo]
        pick = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
        values[:, b * BLOCK:(b + 1) * BLOCK] = torch.where(part < 0, -grid[pick], grid[pick])
    return values, scales


def _exact_value(codes, scales):
    grid = _e4m3_values(codes.device)
    raw = codes.view(torch.uint8).long()
    x = grid[(raw & 127).clamp(max=126)]
    x = torch.where(raw >= 128, -x, x)
    e = scales.view(torch.uint8).double() - 127
    for b in range(-(-x.shape[1] // BLOCK)):
        x[:, b * BLOCK:(b + 1) * BLOCK] *= torch.exp2(e[:, b, None])
    return x


def _pieces(rows, cols):
    step = max(1, (1 << 26) // cols)
    return [(a, min(rows, a + step)) for a in range(0, rows, step)]


def exact(case, seed):
    s = prepare(case, seed)
    op, rows = case["op"], case["rows"]
    if op == "product":
        w = _exact_value(s["w_codes"], s["w_scales"])
        return torch.cat([_exact_value(s["codes"][a:b], s["scales"][a:b]) @ w.t() for a, b in _pieces(rows, case["cols"])])
    if op == "quantize":
        done = [_exact_operand(s["x"][a:b].double()) for a, b in _pieces(rows, case["cols"])]
        return [torch.cat(t) for t in zip(*done)]
    if op == "norm":
        done = []
        for a, b in _pieces(rows, case["cols"]):
            h = s["x"][a:b].double()
            if case["residual"]:   # the sum is held in 16 bits, and what is normalised is what is held
                h = (h + s["residual"][a:b].double()).bfloat16().double()
            y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["cols"] + case["eps"]) * s["weight"].double()
            done.append([*(_exact_operand(y) if case["quantized"] else [y]), h])
        out = [torch.cat(t) for t in zip(*done)]
        return out if case["residual"] else [*out[:-1], None]
    f, size = _frequencies(case)
    hq, hkv, r = case["hq"], case["hkv"], case["dim"]
    x = s["qkv"].view(rows, -1, DIM)
    pos = torch.arange(rows, device=x.device) if s["positions"] is None else s["positions"]
    turned = x[:, :hq + hkv].double()
    for i, freq in enumerate(f):   # each pair as a complex number
        a, b = (2 * i, 2 * i + 1) if case["layout"] == "interleaved" else (i, i + r // 2)
        z = torch.complex(turned[..., a], turned[..., b]) * torch.polar(torch.full_like(pos, size, dtype=torch.float64), pos.double() * freq)[:, None]
        turned[..., a], turned[..., b] = z.real, z.imag
    return [turned[:, :hq], turned[:, hq:], x[:, hq + hkv:].double()]
