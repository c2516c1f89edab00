"""The K/V cache of the answering phase: 8-bit pages, their bookkeeping and attention over them.

CrispCache holds the tensors of one cache (include/crisp.h, `crisp_cache`) and its two workspaces and passes pointers
to libcrisp.so.  Nothing is computed in Python and nothing waits for the device, except poll().
"""
from __future__ import annotations

import ctypes
import operator
from typing import Optional

import torch

from . import binding as B

PAGE = 128
_FORMATS = {"e4m3": B.CACHE_E4M3, "int8": B.CACHE_INT8}


class CrispCache:
    """A paged 8-bit K/V cache over tensors that the caller (or `allocate`) provides.

    k_codes, v_codes  uint8 [layers, pages, kv_heads, 128, 128]: one byte per element, `fmt` "e4m3" or "int8"
    k_scale, v_scale  float32 [layers, pages, kv_heads]: powers of two
    page_table        int32 [max_seqs, max_pages];  seq_lens int32 [max_seqs];  page_refs int32 [pages]

    Lists of sequences are int32 tensors on the cache's device (negative entries are padding).  All calls enqueue on
    `stream` (a torch stream or its handle; default: the current stream of the cache's device) and may be captured into a
    CUDA graph; mistakes that only the device can see (no free page, a sequence listed twice, ...) are raised by poll().
    Calls of one object must not overlap in time (they share its workspaces): use one stream, or order the streams with
    events, also behind the object's creation, which initialises its tensors on the current stream.  Objects over the same
    tensors may read them (attention) at the same time.  Tensors given to a call may be dropped right behind it, whatever its
    stream; the cache itself is kept until its calls have run.
    """

    def __init__(self, k_codes, v_codes, k_scale, v_scale, page_table, seq_lens, page_refs, *, fmt: str = "e4m3"):
        if fmt not in _FORMATS:
            raise ValueError(f"fmt must be one of {sorted(_FORMATS)}, not {fmt!r}")
        if k_codes.dim() != 5 or k_codes.shape[3:] != (PAGE, 128):
            raise ValueError("k_codes must be [layers, pages, kv_heads, 128, 128]")
        self.fmt, self.device = fmt, k_codes.device
        if self.device.type != "cuda":
            raise RuntimeError("CrispCache needs CUDA tensors (no CPU fallback)")
        layers, pages, heads = k_codes.shape[:3]
        max_seqs, max_pages = page_table.shape
        for name, t, shape, dtype in (
                ("k_codes", k_codes, k_codes.shape, torch.uint8), ("v_codes", v_codes, k_codes.shape, torch.uint8),
                ("k_scale", k_scale, (layers, pages, heads), torch.float32),
                ("v_scale", v_scale, (layers, pages, heads), torch.float32),
                ("page_table", page_table, (max_seqs, max_pages), torch.int32),
                ("seq_lens", seq_lens, (max_seqs,), torch.int32), ("page_refs", page_refs, (pages,), torch.int32)):
            self._check(name, t, dtype)
            if tuple(t.shape) != tuple(shape):
                raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
        self.k_codes, self.v_codes, self.k_scale, self.v_scale = k_codes, v_codes, k_scale, v_scale
        self.page_table, self.seq_lens, self.page_refs = page_table, seq_lens, page_refs
        self.n_layers, self.n_pages, self.n_kv_heads = layers, pages, heads
        self.desc = B.CrispCacheDesc(ctypes.sizeof(B.CrispCacheDesc), _FORMATS[fmt], layers, heads, pages, max_seqs,
                                     max_pages, 128, *(t.data_ptr() for t in (
                                         k_codes, v_codes, k_scale, v_scale, page_table, seq_lens, page_refs)))
        pages_ws, attention_ws = B.crisp_cache_workspace_bytes(self.desc)
        self.pages_ws, self.attention_ws = (torch.empty(n, dtype=torch.uint8, device=self.device)
                                            for n in (pages_ws, attention_ws))
        for ws in (self.pages_ws, self.attention_ws):
            ws[:256].zero_()   # status words: the calls only set them
        self._pages_ws, self._attention_ws = ((ws.data_ptr(), ws.numel()) for ws in (self.pages_ws, self.attention_ws))
        self._c, self._lib = ctypes.byref(self.desc), B.load()

    @classmethod
    def allocate(cls, n_pages: int, n_kv_heads: int, max_seqs: int, max_pages: int, *, n_layers: int = 1,
                 fmt: str = "e4m3", device="cuda") -> "CrispCache":
        """An empty cache with tensors of its own."""
        if not torch.cuda.is_available():
            raise RuntimeError("CrispCache needs a CUDA device (no CPU fallback)")
        shape = (n_layers, n_pages, n_kv_heads)
        codes = [torch.empty(*shape, PAGE, 128, dtype=torch.uint8, device=device) for _ in range(2)]
        scale = [torch.empty(shape, dtype=torch.float32, device=device) for _ in range(2)]
        table = torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=device)
        lens, refs = (torch.zeros(n, dtype=torch.int32, device=device) for n in (max_seqs, n_pages))
        return cls(*codes, *scale, table, lens, refs, fmt=fmt)

    # ---- argument checks (host side: types, shapes and places; the device checks the contents)
    def _check(self, name, t, dtype):
        if t.dtype is not dtype or t.device != self.device or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor on {self.device}")

    def _list(self, name, t, n=None):
        """Pointer of an int32 list (None: null)."""
        if t is None:
            return None
        self._check(name, t, torch.int32)
        if t.dim() != 1 or (n is not None and t.shape[0] != n):
            raise ValueError(f"{name} must be one-dimensional" + ("" if n is None else f" with {n} entries"))
        return t.data_ptr()

    def _tokens(self, name, t, tokens, heads):
        """Pointer of a [tokens, heads, 128] bf16 tensor."""
        self._check(name, t, torch.bfloat16)
        if t.shape != (tokens, heads, 128):
            raise ValueError(f"{name} must be [{tokens}, {heads}, 128]")
        return t.data_ptr()

    def check_tokens(self, k, v, tokens):
        """Raises what append would unless k and v are [tokens, kv_heads, 128] bf16 tensors that it takes."""
        if any(self._tokens(name, t, tokens, self.n_kv_heads) % 16 for name, t in (("k", k), ("v", v))):
            raise B.CrispError(B.ERR_INVALID_ARG, "crisp_cache_append")

    def check_append(self, tokens, n_kv_heads, seq_ids, cu_tokens=None, n_new=None, layer=0) -> int:
        """Raises what reserve and append would on the host for that many tokens of n_kv_heads heads, whose K and V need not be
        there yet: nothing is enqueued.  Returns the layer as a number that the calls take."""
        layer = operator.index(layer)
        if n_kv_heads != self.n_kv_heads:
            raise ValueError(f"k and v must have {self.n_kv_heads} heads, not {n_kv_heads}")
        self._list("seq_ids", seq_ids)
        batch = seq_ids.shape[0]
        self._list("cu_tokens", cu_tokens, batch + 1)
        self._list("n_new", n_new, batch)
        if batch > B.CACHE_MAX_BATCH:
            raise B.CrispError(B.ERR_UNSUPPORTED, "crisp_cache_append")
        if not 0 <= layer < self.n_layers or (batch > 0 and cu_tokens is None and tokens % batch != 0):
            raise B.CrispError(B.ERR_INVALID_ARG, "crisp_cache_append")
        return layer

    def check_attention(self, tokens, n_q_heads, seq_ids, cu_tokens=None, max_new: Optional[int] = None) -> int:
        """The same for attention of that many tokens of n_q_heads heads, where check_append has passed.  Returns max_new."""
        batch = seq_ids.shape[0]
        max_new = self._max_new(tokens, batch, cu_tokens) if max_new is None else operator.index(max_new)
        per = tokens // batch if batch > 0 and cu_tokens is None else 0
        if not per <= max_new < 1 << 31 or n_q_heads <= 0 or n_q_heads % self.n_kv_heads != 0:
            raise B.CrispError(B.ERR_INVALID_ARG, "crisp_cache_attention")
        if n_q_heads // self.n_kv_heads > B.MAX_GROUP:
            raise B.CrispError(B.ERR_UNSUPPORTED, "crisp_cache_attention")
        return max_new

    @staticmethod
    def _max_new(tokens, batch, cu_tokens):
        """The items' largest number of tokens that the shapes allow."""
        return tokens if cu_tokens is not None or batch == 0 else tokens // batch

    def _call(self, name, stream, *args):
        """The C call of that name on (cache, *args, stream), with the cache's device current.  (The answering loop calls
        this once or more per layer and token, so the way to the library is kept short.)"""
        index = self.device.index
        if stream is None:
            stream = torch._C._cuda_getCurrentRawStream(index)
        elif not isinstance(stream, int):
            stream = stream.cuda_stream
        if torch.cuda.current_device() == index:
            rc = getattr(self._lib, name)(self._c, *args, stream)
        else:
            with torch.cuda.device(index):
                rc = getattr(self._lib, name)(self._c, *args, stream)
        if rc != B.OK:
            raise B.CrispError(rc, name)

    # ---- pages
    def reserve(self, seq_ids, n_new: Optional[torch.Tensor] = None, stream=None) -> None:
        """Adds n_new[i] (None: one) tokens to sequence seq_ids[i] and gives it the pages for them.  All or nothing; while
        a refused call stands (until one that lists the sequence succeeds), append leaves the sequence as it is."""
        ids, n = self._list("seq_ids", seq_ids), seq_ids.shape[0]
        self._call("crisp_cache_reserve", stream, ids, self._list("n_new", n_new, n), n, *self._pages_ws)
        self._used(stream, seq_ids, n_new)

    def fork(self, src, dst, n_tokens: Optional[torch.Tensor] = None, share: bool = True, stream=None) -> None:
        """Makes the empty sequence dst[i] the first n_tokens[i] (None: all) tokens of src[i]."""
        n = src.shape[0]
        self._call("crisp_cache_fork", stream, self._list("src", src), self._list("dst", dst, n),
                   self._list("n_tokens", n_tokens, n), n, 1 if share else 0, *self._pages_ws)
        self._used(stream, src, dst, n_tokens)

    def free(self, seq_ids, stream=None) -> None:
        """Empties the listed sequences."""
        self._call("crisp_cache_free", stream, self._list("seq_ids", seq_ids), seq_ids.shape[0], *self._pages_ws)
        self._used(stream, seq_ids)

    def compact(self, n_used: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Moves the pages in use to the front of the pool; returns how many there are (int32 [1], on the device)."""
        if n_used is None:
            n_used = self._new((1,), torch.int32, stream)
        self._call("crisp_cache_compact", stream, self._list("n_used", n_used, 1), *self._pages_ws)
        self._used(stream, n_used)
        return n_used

    # ---- contents
    def append(self, k, v, seq_ids, cu_tokens: Optional[torch.Tensor] = None, layer: int = 0, stream=None) -> None:
        """Writes the last tokens of the listed sequences, packed in k and v [tokens, kv_heads, 128] bf16: item i owns
        tokens cu_tokens[i] .. cu_tokens[i + 1] - 1 (None: the same number for every item)."""
        n, batch = k.shape[0], seq_ids.shape[0]
        self._call("crisp_cache_append", stream, layer, self._list("seq_ids", seq_ids),
                   self._list("cu_tokens", cu_tokens, batch + 1), batch, n, self._tokens("k", k, n, self.n_kv_heads),
                   self._tokens("v", v, n, self.n_kv_heads), *self._pages_ws)
        self._used(stream, k, v, seq_ids, cu_tokens)

    def attention(self, q, seq_ids, cu_tokens: Optional[torch.Tensor] = None, max_new: Optional[int] = None,
                  layer: int = 0, softmax_scale: float = 0.0, o: Optional[torch.Tensor] = None,
                  lse: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Causal attention of the newest tokens, q [tokens, q_heads, 128] bf16 packed as in append, over everything
        their sequences hold.  max_new: a bound on the items' numbers of tokens (None: what the shapes allow); it picks
        the kernel, so a server that answers token by token with cu_tokens should give it.
        lse: optional float32 [q_heads, tokens].  Returns o like q."""
        if q.dim() != 3:
            raise ValueError("q must be [tokens, q_heads, 128]")
        n, hq, _ = q.shape
        batch = seq_ids.shape[0]
        pq, ids, cu = self._tokens("q", q, n, hq), self._list("seq_ids", seq_ids), self._list("cu_tokens", cu_tokens, batch + 1)
        if max_new is None:
            max_new = self._max_new(n, batch, cu_tokens)
        plse = None
        if lse is not None:
            self._check("lse", lse, torch.float32)
            if lse.shape != (hq, n):
                raise ValueError(f"lse must be [{hq}, {n}]")
            plse = lse.data_ptr()
        if o is not None:
            po = self._tokens("o", o, n, hq)
            given = o
        else:
            o = torch.empty_like(q) if stream is None else self._new(q.shape, torch.bfloat16, stream)
            po = o.data_ptr()
            given = None
        self._call("crisp_cache_attention", stream, layer, ids, cu, batch, n, max_new, hq, softmax_scale, pq, po, plse,
                   *self._attention_ws)
        self._used(stream, q, seq_ids, cu_tokens, given, lse)
        return o

    def _torch_stream(self, stream):
        """The torch stream of a stream or handle.  (0 is the default stream's; ExternalStream(0) would be a new one.)"""
        if not isinstance(stream, int):
            return stream
        return torch.cuda.ExternalStream(stream, device=self.device) if stream else torch.cuda.default_stream(self.device)

    def _used(self, stream, *tensors):
        """Tells the allocator that a call on this stream uses these tensors, so that their memory is not handed out again before
        it has run."""
        if stream is None:   # (compiled: an answer comes here three times per layer and token)
            B.calls().used(self.device.index, *tensors)
            return
        stream = self._torch_stream(stream)
        for t in tensors:
            if t is not None:
                t.record_stream(stream)

    def _new(self, shape, dtype, stream):
        """An output, allocated on the stream that will write it (memory that the current stream freed may still be in
        use there)."""
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self._torch_stream(stream)):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def poll(self, stream=None) -> None:
        """Waits for the stream and raises the first error that the device has recorded since the last poll: that of the
        pages' calls, or attention's.  With one of each, the message names both."""
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        with torch.cuda.device(self.device):
            pages, attention = (B.crisp_poll_device_status(ws, stream) for ws in (self.pages_ws, self.attention_ws))
        if pages != B.OK and attention != B.OK:
            raise B.CrispError(pages, f"cache status (attention: {B.status_string(attention)} ({attention}); pages)")
        B.check(pages, "cache status (pages)")
        B.check(attention, "cache status (attention)")
