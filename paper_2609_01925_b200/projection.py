"""The way into and out of a layer's attention: norm, 8-bit products, rotary positions, and CrispAttention, which runs them
around CrispLayer (a prompt) and CrispCache (the answer).

An operand of a product is a pair (codes, scales): float8_e4m3fn [rows, columns] and float8_e8m0fnu
[rows, 4 ceil(columns / 512)], one power-of-two scale for each row and 128 columns (include/crisp.h, `crisp_quantize`).
Nothing is computed in Python and nothing waits for the device, except poll().  All calls enqueue on `stream` (a torch stream
or its handle; default: the current stream of the tensors' device) and may be captured into a CUDA graph; tensors given to a
call may be dropped right behind it, whatever its stream.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import binding as B
from .cache import CrispCache
from .layer import CrispLayer

HEAD = 128
CODES, SCALES = torch.float8_e4m3fn, torch.float8_e8m0fnu
_LAYOUTS = {"half": B.ROTARY_HALF, "interleaved": B.ROTARY_INTERLEAVED}
_SCALINGS = {"none": B.ROTARY_PLAIN, "linear": B.ROTARY_LINEAR, "base": B.ROTARY_BASE, "ramp": B.ROTARY_RAMP,
             "bands": B.ROTARY_BANDS}


# (Argument checks, outputs and streams of these calls are in csrc/calls.cpp.)
def _scale_cols(cols):
    return (cols + 511) // 512 * 4


# ---- rows
def quantize(x, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """bf16 [rows, columns] as an operand (codes, scales): weights, once, or the output of attention."""
    return B.calls().quantize(x, stream)


def rms_norm(x, weight=None, residual=None, *, eps: float = 1e-5, sum_out: Optional[torch.Tensor] = None, stream=None):
    """Root-mean-square norm of bf16 rows: h = x + residual (rounded to bf16; without one h is x),
    y = h / sqrt(mean(h^2) + eps) * weight.  Returns (y, h), h None without a residual.  sum_out: where h goes; it may be x
    or residual."""
    return B.calls().rms_norm(x, weight, residual, eps, sum_out, False, stream)


def rms_norm_quantize(x, weight=None, residual=None, *, eps: float = 1e-5, sum_out: Optional[torch.Tensor] = None, stream=None):
    """rms_norm with y as an operand of a product: returns (codes, scales, h)."""
    return B.calls().rms_norm(x, weight, residual, eps, sum_out, True, stream)


# ---- products
class CrispLinear:
    """Weights [out_features, in_features] as an operand, and products with them.

    Products of one object may overlap, on any streams (they share a status word only), behind the object's creation, which
    zeroes that word on the current stream.  The object is kept until its calls have run.
    """

    def __init__(self, codes, scales):
        if not codes.is_cuda:
            raise RuntimeError("codes must be a CUDA tensor (no CPU fallback)")
        if codes.dim() != 2 or codes.dtype is not CODES or not codes.is_contiguous():
            raise ValueError(f"codes must be a contiguous {CODES} matrix")
        self.n_out, self.n_in = codes.shape
        shape = (self.n_out, _scale_cols(self.n_in))
        if scales.dtype is not SCALES or scales.device != codes.device or not scales.is_contiguous() or scales.shape != shape:
            raise ValueError(f"scales must be a contiguous {SCALES} tensor of shape {shape} beside the codes")
        self.codes, self.scales, self.device = codes, scales, codes.device
        self.ws = torch.zeros(B.crisp_matmul_workspace_bytes(), dtype=torch.uint8, device=self.device)

    @classmethod
    def from_weight(cls, weight) -> "CrispLinear":
        """From bf16 weights [out_features, in_features], converted here, once."""
        return cls(*quantize(weight))

    def __call__(self, codes, scales, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """bf16 [rows, out_features]: the operand's rows times the transposed weights."""
        return B.calls().matmul(codes, scales, self.codes, self.scales, self.ws, out, stream)

    def poll(self, stream=None) -> None:
        """Waits for the stream and raises the first error that the device has recorded since the last poll."""
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        with torch.cuda.device(self.device):
            B.check(B.crisp_poll_device_status(self.ws, stream), "product status")


# ---- rotary positions
class CrispRotary:
    """Rotary positions with frequencies theta^(-2 i / rotary_dim) (include/crisp.h, `crisp_rotary_init`).

    layout   "half" (pairs i, i + rotary_dim / 2) or "interleaved" (pairs 2 i, 2 i + 1); the rest of a head is copied
    scaling  for lengths beyond `original`: "none", "linear", "base", "ramp" or "bands", by `factor`; low, high: the turns
             between which "ramp" and "bands" pass from one frequency to the other (None: 1 and 32, 1 and 4)
    magnitude  factor on what is rotated (None: 1, and 0.1 ln(factor) + 1 for "ramp")
    """

    def __init__(self, theta: float, *, rotary_dim: int = HEAD, layout: str = "half", scaling: str = "none", factor: float = 1.0,
                 original: int = 0, low: Optional[float] = None, high: Optional[float] = None,
                 magnitude: Optional[float] = None):
        if layout not in _LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(_LAYOUTS)}, not {layout!r}")
        if scaling not in _SCALINGS:
            raise ValueError(f"scaling must be one of {sorted(_SCALINGS)}, not {scaling!r}")
        if any(turns is not None and not turns > 0 for turns in (low, high)):
            raise ValueError("low and high must be positive")   # (zero stands for the usual turns in the C call)
        self.plan = B.crisp_rotary_init(rotary_dim, _LAYOUTS[layout], theta, _SCALINGS[scaling], factor, original, low or 0.0,
                                        high or 0.0)
        if magnitude is not None:
            self.plan.magnitude = magnitude

    def split(self, qkv, n_q_heads: int, n_kv_heads: int, positions: Optional[torch.Tensor] = None, *, first_position: int = 0,
              stream=None):
        """q [tokens, n_q_heads, 128], k and v [tokens, n_kv_heads, 128] from a product's rows
        [tokens, (n_q_heads + 2 n_kv_heads) 128]: q and k rotated, v copied.  positions: int32 [tokens] (None: first_position,
        first_position + 1, ...)."""
        return B.calls().rotary_split(ctypes.addressof(self.plan), qkv, n_q_heads, n_kv_heads, positions, first_position, stream)

    def rotate(self, x, positions: Optional[torch.Tensor] = None, *, first_position: int = 0,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """bf16 x [tokens, heads, 128], whose tokens may have any stride, rotated.  out: contiguous; it may be x."""
        return B.calls().rotary_rotate(ctypes.addressof(self.plan), x, positions, first_position, out, stream)


# ---- a layer's attention, from hidden states to hidden states
class CrispAttention:
    """The attention part of a layer: norm (with the residual's addition), Q/K/V product, rotary positions, attention, output
    product.

    qkv   CrispLinear with (n_q_heads + 2 n_kv_heads) 128 outputs, in the order q, k, v
    out   CrispLinear from n_q_heads 128 inputs
    """

    def __init__(self, qkv: CrispLinear, out: CrispLinear, rotary: CrispRotary, n_q_heads: int, n_kv_heads: int, *,
                 norm_weight: Optional[torch.Tensor] = None, eps: float = 1e-5):
        if qkv.n_out != (n_q_heads + 2 * n_kv_heads) * HEAD or out.n_in != n_q_heads * HEAD or qkv.device != out.device:
            raise ValueError("qkv must have (n_q_heads + 2 n_kv_heads) 128 outputs and out n_q_heads 128 inputs, on one device")
        self.qkv, self.out, self.rotary, self.norm_weight, self.eps = qkv, out, rotary, norm_weight, eps
        self.n_q_heads, self.n_kv_heads = n_q_heads, n_kv_heads

    def project(self, x, residual=None, positions=None, *, first_position: int = 0, stream=None):
        """(q, k, v, h) of hidden states x [tokens, in_features]; h = x + residual (None without one)."""
        codes, scales, h = rms_norm_quantize(x, self.norm_weight, residual, eps=self.eps, stream=stream)
        qkv = self.qkv(codes, scales, stream=stream)
        return (*self.rotary.split(qkv, self.n_q_heads, self.n_kv_heads, positions, first_position=first_position,
                                   stream=stream), h)

    def finish(self, o, stream=None) -> torch.Tensor:
        """The output product of attention's o [tokens, n_q_heads, 128]."""
        return self.out(*quantize(o.view(o.shape[0], self.n_q_heads * HEAD), stream=stream), stream=stream)

    def _same_device(self, cache):
        if cache.device != self.qkv.device:
            raise ValueError(f"the cache must be on {self.qkv.device}")

    def prompt(self, x, layer: CrispLayer, residual=None, *, cache: Optional[CrispCache] = None, seq_ids=None,
               cache_layer: int = 0, dense_below_tokens: int = 0, stream=None):
        """A whole prompt: x [layer.p.seq_len, in_features] through CrispLayer.forward; with a cache its K and V are kept there
        (CrispLayer.store).  Returns (out, h)."""
        # (the attention is given pointers and takes sizes from layer.p: all of this comes before the first launch)
        p = layer.p
        if x.dim() != 2 or x.shape[0] != p.seq_len:
            raise ValueError(f"x must be [{p.seq_len}, {self.qkv.n_in}], the layer's tokens")
        if (p.n_q_heads, p.n_kv_heads) != (self.n_q_heads, self.n_kv_heads) or layer.o.device != self.qkv.device:
            raise ValueError(f"the layer must have {self.n_q_heads} / {self.n_kv_heads} heads and be on {self.qkv.device}")
        if cache is not None:
            if seq_ids is None or seq_ids.shape != (1,):
                raise ValueError("seq_ids must name one sequence")
            self._same_device(cache)
            cache_layer = cache.check_append(p.seq_len, self.n_kv_heads, seq_ids, layer=cache_layer)
        q, k, v, h = self.project(x, residual, stream=stream)
        o = layer.forward(q, k, v, stream=stream, dense_below_tokens=dense_below_tokens)
        if cache is not None:
            layer.store(k, v, cache, seq_ids, cache_layer, stream=stream)
        return self.finish(o, stream), h

    def answer(self, x, positions, cache: CrispCache, seq_ids, residual=None, *, cu_tokens=None, n_new=None,
               max_new: Optional[int] = None, cache_layer: int = 0, stream=None):
        """New tokens of cached sequences, packed in x as in CrispCache.append, at their positions (int32 [tokens]): appended
        and attended to.  At cache_layer 0 the sequences grow by n_new (None: one token each).  Returns (out, h)."""
        # (all that append and attention refuse on the host, before the sequences grow: tokens that are counted and not written
        # would be read as they are)
        if x.dim() != 2:
            raise ValueError(f"x must be [tokens, {self.qkv.n_in}]")
        self._same_device(cache)
        tokens = x.shape[0]
        cache_layer = cache.check_append(tokens, self.n_kv_heads, seq_ids, cu_tokens, n_new, cache_layer)
        max_new = cache.check_attention(tokens, self.n_q_heads, seq_ids, cu_tokens, max_new)
        if cache_layer == 0 and n_new is None and cu_tokens is None and tokens != seq_ids.shape[0]:
            raise ValueError("without n_new there must be one token for each sequence")
        q, k, v, h = self.project(x, residual, positions, stream=stream)
        if cache_layer == 0:
            cache.reserve(seq_ids, n_new, stream)
        cache.append(k, v, seq_ids, cu_tokens, layer=cache_layer, stream=stream)
        o = cache.attention(q, seq_ids, cu_tokens, max_new, layer=cache_layer, stream=stream)
        return self.finish(o, stream), h

    def poll(self, stream=None) -> None:
        for linear in (self.qkv, self.out):
            linear.poll(stream)
