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


# ---- what the calls below share (an answer calls them several times per layer and token, so the way to the library is kept
# short: places are device indexes, -1 for the CPU, and outputs are made beside a tensor that is there)
_BF16, _I32 = torch.bfloat16, torch.int32


def _check(name, t, dtype, index, shape=None):
    """Pointer of a contiguous tensor of that type, place and shape."""
    if t.dtype is not dtype or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on cuda:{index}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    return t.data_ptr()


def _rows(name, t, dtype):
    """Place and shape of a matrix of that type."""
    index, shape = t.get_device(), t.shape
    if index < 0:
        raise RuntimeError(f"{name} must be a CUDA tensor (no CPU fallback)")
    if len(shape) != 2 or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} matrix")
    return index, shape


def _scale_cols(cols):
    return (cols + 511) // 512 * 4


def _torch_stream(stream, index):
    """The torch stream of a stream or handle.  (0 is the default stream's; ExternalStream(0) would be a new one.)"""
    if not isinstance(stream, int):
        return stream
    return torch.cuda.ExternalStream(stream, device=index) if stream else torch.cuda.default_stream(index)


def _new(like, shape, dtype, stream):
    """An output beside `like`, allocated on the stream that will write it."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(_torch_stream(stream, like.get_device())):
        return like.new_empty(shape, dtype=dtype)


def _new_like(like, dtype, stream):
    """The same with the shape of `like`."""
    if stream is None:
        return torch.empty_like(like, dtype=dtype)
    return _new(like, like.shape, dtype, stream)


def _call(name, index, stream, args, tensors):
    """The C call of that name on (*args, stream), with device `index` current."""
    function = getattr(B.load(), name)
    if stream is None:
        raw = torch._C._cuda_getCurrentRawStream(index)
    else:
        raw = stream if isinstance(stream, int) else stream.cuda_stream
    if torch._C._cuda_getDevice() == index:
        rc = function(*args, raw)
    else:
        with torch.cuda.device(index):
            rc = function(*args, raw)
    if rc != B.OK:
        raise B.CrispError(rc, name)
    if stream is not None:
        stream = _torch_stream(stream, index)
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


# ---- rows
def quantize(x, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """bf16 [rows, columns] as an operand (codes, scales): weights, once, or the output of attention."""
    index, (rows, cols) = _rows("x", x, _BF16)
    codes, scales = _new_like(x, CODES, stream), _new(x, (rows, _scale_cols(cols)), SCALES, stream)
    _call("crisp_quantize", index, stream, (x.data_ptr(), rows, cols, codes.data_ptr(), scales.data_ptr()), (x, codes, scales))
    return codes, scales


def _norm_inputs(x, weight, residual, sum_out, stream):
    """(place, shape, pointers of residual, weight and sum, sum)."""
    index, shape = _rows("x", x, _BF16)
    w = None if weight is None else _check("weight", weight, _BF16, index, shape[1:])
    if residual is None:
        if sum_out is not None:
            raise ValueError("sum_out belongs to a residual")
        return index, shape, None, w, None, None
    r = _check("residual", residual, _BF16, index, shape)
    if sum_out is None:
        sum_out = _new_like(x, _BF16, stream)
        return index, shape, r, w, sum_out.data_ptr(), sum_out
    return index, shape, r, w, _check("sum_out", sum_out, _BF16, index, shape), sum_out


def rms_norm(x, weight=None, residual=None, *, eps: float = 1e-5, sum_out: Optional[torch.Tensor] = None, stream=None):
    """Root-mean-square norm of bf16 rows: h = x + residual (rounded to bf16; without one h is x),
    y = h / sqrt(mean(h^2) + eps) * weight.  Returns (y, h), h None without a residual.  sum_out: where h goes; it may be x
    or residual."""
    index, (rows, cols), r, w, total, h = _norm_inputs(x, weight, residual, sum_out, stream)
    y = _new_like(x, _BF16, stream)
    _call("crisp_rms_norm", index, stream, (x.data_ptr(), r, w, rows, cols, eps, total, y.data_ptr(), None, None),
          (x, weight, residual, h, y))
    return y, h


def rms_norm_quantize(x, weight=None, residual=None, *, eps: float = 1e-5, sum_out: Optional[torch.Tensor] = None, stream=None):
    """rms_norm with y as an operand of a product: returns (codes, scales, h)."""
    index, (rows, cols), r, w, total, h = _norm_inputs(x, weight, residual, sum_out, stream)
    codes, scales = _new_like(x, CODES, stream), _new(x, (rows, _scale_cols(cols)), SCALES, stream)
    _call("crisp_rms_norm", index, stream,
          (x.data_ptr(), r, w, rows, cols, eps, total, None, codes.data_ptr(), scales.data_ptr()),
          (x, weight, residual, h, codes, scales))
    return codes, scales, h


# ---- products
class CrispLinear:
    """Weights [out_features, in_features] as an operand, and products with them."""

    def __init__(self, codes, scales):
        self._index, (self.n_out, self.n_in) = _rows("codes", codes, CODES)
        self._cols = _scale_cols(self.n_in)
        _check("scales", scales, SCALES, self._index, (self.n_out, self._cols))
        self.codes, self.scales, self.device = codes, scales, codes.device
        self.ws = torch.zeros(B.crisp_matmul_workspace_bytes(), dtype=torch.uint8, device=self.device)
        self._w, self._ws = (codes.data_ptr(), scales.data_ptr()), (self.ws.data_ptr(), self.ws.numel())

    @classmethod
    def from_weight(cls, weight) -> "CrispLinear":
        """From bf16 weights [out_features, in_features], converted here, once."""
        return cls(*quantize(weight))

    def __call__(self, codes, scales, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """bf16 [rows, out_features]: the operand's rows times the transposed weights."""
        index, (rows, cols) = _rows("codes", codes, CODES)
        if cols != self.n_in or index != self._index:
            raise ValueError(f"codes must have {self.n_in} columns and be on {self.device}")
        ps = _check("scales", scales, SCALES, index, (rows, self._cols))
        if out is None:
            out = _new(codes, (rows, self.n_out), _BF16, stream)
            po = out.data_ptr()
        else:
            po = _check("out", out, _BF16, index, (rows, self.n_out))
        _call("crisp_matmul", index, stream, (codes.data_ptr(), ps, *self._w, rows, self.n_out, cols, po, *self._ws),
              (codes, scales, self.codes, self.scales, self.ws, out))
        return out

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
        self.plan = B.crisp_rotary_init(rotary_dim, _LAYOUTS[layout], theta, _SCALINGS[scaling], factor, original, low or 0.0,
                                        high or 0.0)
        if magnitude is not None:
            self.plan.magnitude = magnitude
        self._plan = ctypes.byref(self.plan)

    def split(self, qkv, n_q_heads: int, n_kv_heads: int, positions: Optional[torch.Tensor] = None, *, first_position: int = 0,
              stream=None):
        """q [tokens, n_q_heads, 128], k and v [tokens, n_kv_heads, 128] from a product's rows
        [tokens, (n_q_heads + 2 n_kv_heads) 128]: q and k rotated, v copied.  positions: int32 [tokens] (None: first_position,
        first_position + 1, ...)."""
        index, shape = qkv.get_device(), qkv.shape
        if index < 0:
            raise RuntimeError("qkv must be a CUDA tensor (no CPU fallback)")
        if n_q_heads <= 0 or n_kv_heads <= 0:
            raise ValueError("there must be heads")
        if len(shape) != 2 or shape[1] != (n_q_heads + 2 * n_kv_heads) * HEAD or qkv.dtype is not _BF16 or qkv.stride(1) != 1:
            raise ValueError(f"qkv must be bf16 [tokens, {(n_q_heads + 2 * n_kv_heads) * HEAD}] with contiguous rows")
        n, row = shape
        if n > 1:
            row = qkv.stride(0)
        q, k = _new(qkv, (n, n_q_heads, HEAD), _BF16, stream), _new(qkv, (n, n_kv_heads, HEAD), _BF16, stream)
        v = _new_like(k, _BF16, stream)
        if n:
            at = qkv.data_ptr()
            at_k = at + 2 * HEAD * n_q_heads
            _call("crisp_rotary", index, stream,
                  (self._plan, n, None if positions is None else _check("positions", positions, _I32, index, (n,)), first_position,
                   n_q_heads, n_kv_heads, at, row, at_k, row, at_k + 2 * HEAD * n_kv_heads, row, q.data_ptr(), k.data_ptr(),
                   v.data_ptr()), (qkv, positions, q, k, v))
        return q, k, v

    def rotate(self, x, positions: Optional[torch.Tensor] = None, *, first_position: int = 0,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """bf16 x [tokens, heads, 128], whose tokens may have any stride, rotated.  out: contiguous; it may be x."""
        index, shape = x.get_device(), x.shape
        if index < 0:
            raise RuntimeError("x must be a CUDA tensor (no CPU fallback)")
        if (len(shape) != 3 or x.dtype is not _BF16 or shape[1] == 0 or shape[2] != HEAD or x.stride(2) != 1
                or (shape[1] > 1 and x.stride(1) != HEAD)):
            raise ValueError("x must be bf16 [tokens, heads, 128] with contiguous tokens")
        n, heads, _ = shape
        if out is None:
            out = _new(x, shape, _BF16, stream)
        po = _check("out", out, _BF16, index, shape)
        if n:
            _call("crisp_rotary", index, stream,
                  (self._plan, n, None if positions is None else _check("positions", positions, _I32, index, (n,)), first_position,
                   heads, 0, x.data_ptr(), x.stride(0) if n > 1 else heads * HEAD, None, 0, None, 0, po, None, None),
                  (x, positions, out))
        return out


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

    def prompt(self, x, layer: CrispLayer, residual=None, *, cache: Optional[CrispCache] = None, seq_ids=None,
               cache_layer: int = 0, dense_below_tokens: int = 0, stream=None):
        """A whole prompt: x [layer.p.seq_len, in_features] through CrispLayer.forward; with a cache its K and V are kept there
        (CrispLayer.store).  Returns (out, h)."""
        q, k, v, h = self.project(x, residual, stream=stream)
        o = layer.forward(q, k, v, stream=stream, dense_below_tokens=dense_below_tokens)
        if cache is not None:
            layer.store(k, v, cache, seq_ids, cache_layer, stream=stream)
        return self.finish(o, stream), h

    def answer(self, x, positions, cache: CrispCache, seq_ids, residual=None, *, cu_tokens=None, n_new=None,
               max_new: Optional[int] = None, cache_layer: int = 0, stream=None):
        """New tokens of cached sequences, packed in x as in CrispCache.append, at their positions (int32 [tokens]): appended
        and attended to.  At cache_layer 0 the sequences grow by n_new (None: one token each).  Returns (out, h)."""
        q, k, v, h = self.project(x, residual, positions, stream=stream)
        if cache_layer == 0:
            cache.reserve(seq_ids, n_new, stream)
        cache.append(k, v, seq_ids, cu_tokens, layer=cache_layer, stream=stream)
        o = cache.attention(q, seq_ids, cu_tokens, max_new, layer=cache_layer, stream=stream)
        return self.finish(o, stream), h

    def poll(self, stream=None) -> None:
        for linear in (self.qkv, self.out):
            linear.poll(stream)
