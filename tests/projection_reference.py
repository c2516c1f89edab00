"""The operators around the attention in float64, straight from their definitions: operands of 8-bit products, the norm,
the product and rotary positions.  Shares no code with the package."""
import math

import numpy as np
import torch

from tests.cache_reference import E4M3

GRID = np.array(E4M3[:127])     # the values of the bytes 0..126, ascending


def scale_cols(cols):
    return -(-cols // 512) * 4


def exponent(amax):
    """Smallest e >= -126 with amax <= 448 2^e."""
    if amax == 0:
        return -126
    m, k = math.frexp(amax)     # amax = m 2^k, 0.5 <= m < 1;  448 = 0.875 2^9
    return max(-126, k - 9 if m <= 0.875 else k - 8)


def encode(v):
    """Bytes of the nearest codes of float64 values, ties to the even one; infinities to the largest, NaN to 0x7f."""
    v = np.asarray(v, np.float64)
    a = np.minimum(np.abs(np.nan_to_num(v, nan=0.0, posinf=1e300, neginf=-1e300)), 448.0)
    hi = np.clip(np.searchsorted(GRID, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = GRID[hi] - a, a - GRID[lo]
    pick = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    out = pick + 128 * np.signbit(v)
    return np.where(np.isnan(v), 0x7f, out).astype(np.uint8)


def quantize(x):
    """(codes, scales) as bytes, of float64 [rows, cols]."""
    rows, cols = x.shape
    codes, scales = np.zeros((rows, cols), np.uint8), np.full((rows, scale_cols(cols)), 127, np.uint8)
    for r in range(rows):
        for b in range(-(-cols // 128)):
            part = x[r, 128 * b:128 * b + 128]
            finite = np.abs(part[np.isfinite(part)])
            e = exponent(finite.max() if finite.size else 0.0)
            codes[r, 128 * b:128 * b + 128] = encode(part * 2.0 ** -e)
            scales[r, b] = e + 127
    return codes, scales


def values(codes, scales):
    """float64 of bytes (NaN codes to NaN)."""
    full = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 128, axis=1)[:, :codes.shape[1]]
    return np.array(E4M3)[codes] * full


def half_step(v):
    """Half the distance between neighbouring e4m3 numbers around |v|, for values in units of the scale."""
    a = np.maximum(np.abs(v), 2.0 ** -6)
    return 2.0 ** (np.floor(np.log2(a)) - 4)


def bf16(x):
    """float64 to bf16 and back, rounded once."""
    x = torch.as_tensor(np.asarray(x, np.float64))
    f = x.float()
    # (float64 -> float32 -> bf16 rounds twice; where the first rounding lands on a tie, move it off it again)
    tie = (f.view(torch.int32) & 0xffff) == 0x8000
    away = torch.where(x.abs() > f.double().abs(), 1, -1).int()
    f = torch.where(tie & (x != f.double()), (f.view(torch.int32) + away).view(torch.float32), f)
    return f.bfloat16().double().numpy()


def norm(x, residual, weight, eps):
    """(y, h) in float64; h is what is stored."""
    h = x if residual is None else bf16(x + residual)
    y = h / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return (y if weight is None else y * weight), h


def frequencies(dim, theta, scaling="none", factor=1.0, original=0, low=None, high=None):
    low = 1.0 if low is None else low
    high = (32.0 if scaling == "ramp" else 4.0) if high is None else high
    if scaling == "base":
        theta = theta * factor ** (dim / (dim - 2))
    f = [theta ** (-2.0 * i / dim) for i in range(dim // 2)]
    if scaling == "linear":
        return [x / factor for x in f]
    if scaling == "bands":
        keep = [(original * x / (2 * math.pi) - low) / (high - low) for x in f]
    elif scaling == "ramp":
        pair = lambda turns: dim * math.log(original / (2 * math.pi * turns)) / (2 * math.log(theta))  # noqa: E731
        a, b = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), dim - 1)
        keep = [1 - (i - a) / max(b - a, 0.001) for i in range(dim // 2)]
    else:
        return f
    keep = [min(max(c, 0.0), 1.0) for c in keep]
    return [x * c + x / factor * (1 - c) for x, c in zip(f, keep)]


def rotate(x, positions, freq, layout, magnitude=1.0):
    """float64 x [tokens, heads, 128]."""
    out, n = x.copy(), len(freq)
    for i, f in enumerate(freq):
        a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + n)
        angle = np.array([float(p) for p in positions]) * f
        z = (x[:, :, a] + 1j * x[:, :, b]) * (magnitude * np.exp(1j * angle))[:, None]
        out[:, :, a], out[:, :, b] = z.real, z.imag
    return out
