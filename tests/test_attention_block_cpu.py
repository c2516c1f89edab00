"""CrispAttention, CrispLayer and CrispCache without a GPU: what they hand to the library, and what they refuse before the first call.
The library and the compiled calls are replaced by stand-ins that write down what they are given; nothing is launched."""
import types

import pytest
import torch

import paper_2609_01925_b200 as crisp
from paper_2609_01925_b200 import binding as B

CPU = torch.device("cpu")
HQ, HKV, HIDDEN = 4, 2, 64


class Calls:
    """Stand-in for the compiled calls: outputs of the right shapes, and a list of what was called."""

    def __init__(self, log):
        self.log = log

    def rms_norm(self, x, weight, residual, eps, sum_out, quantized, stream):
        self.log.append("rms_norm")
        return x, x, None if residual is None else residual

    def matmul(self, codes, scales, w_codes, w_scales, ws, out, stream):
        self.log.append("matmul")
        return torch.zeros(codes.shape[0], w_codes.shape[0], dtype=torch.bfloat16)

    def rotary_split(self, plan, qkv, hq, hkv, positions, first, stream):
        self.log.append("rotary")
        return tuple(torch.zeros(qkv.shape[0], h, 128, dtype=torch.bfloat16) for h in (hq, hkv, hkv))

    def quantize(self, x, stream):
        self.log.append("quantize")
        return x, x


class Library:
    """Stand-in for libcrisp.so's calls of the cache."""

    def __init__(self, log):
        self.log = log

    def __getattr__(self, name):
        return lambda *args: self.log.append(name) or B.OK


def linear(n_out, n_in):
    made = object.__new__(crisp.CrispLinear)
    made.codes, made.scales, made.ws = torch.zeros(n_out, n_in, dtype=torch.uint8), None, None
    made.n_out, made.n_in, made.device = n_out, n_in, CPU
    return made


def make_cache(log, heads=HKV, layers=2, device=CPU):
    cache = object.__new__(crisp.CrispCache)
    cache.device, cache.n_kv_heads, cache.n_layers = device, heads, layers
    cache._pages_ws = cache._attention_ws = (0, 0)
    cache._call = lambda name, stream, *args: log.append(name)
    cache._used = lambda *args: None
    return cache


def make_layer(log, tokens, hq=HQ, hkv=HKV):
    layer = object.__new__(crisp.CrispLayer)
    layer.p = crisp.make_params(tokens, hq, hkv)
    layer.o = torch.zeros(tokens, hq, 128, dtype=torch.bfloat16)
    layer.n_tokens = torch.full((1,), tokens, dtype=torch.int32)
    layer.forward = lambda *args, **kw: log.append("forward") or layer.o
    return layer


@pytest.fixture
def log(monkeypatch):
    made = []
    monkeypatch.setattr(B, "calls", lambda: Calls(made))
    return made


@pytest.fixture
def block():
    return crisp.CrispAttention(linear((HQ + 2 * HKV) * 128, HIDDEN), linear(HIDDEN, HQ * 128), crisp.CrispRotary(1e4), HQ, HKV)


def states(tokens, cols=HIDDEN):
    return torch.zeros(tokens, cols, dtype=torch.bfloat16)


def ids(*which):
    return torch.tensor(which, dtype=torch.int32)


# ------------------------------------------------------------------------------------------------ a prompt
def test_prompt_calls(log, block):
    block.prompt(states(300), make_layer(log, 300))
    assert log == ["rms_norm", "matmul", "rotary", "forward", "quantize", "matmul"]
    log.clear()
    block.prompt(states(300), make_layer(log, 300), cache=make_cache(log), seq_ids=ids(1))
    assert log == ["rms_norm", "matmul", "rotary", "forward", "crisp_cache_reserve", "crisp_cache_append", "quantize", "matmul"]
    log.clear()
    block.prompt(states(300), make_layer(log, 300), cache=make_cache(log), seq_ids=ids(1), cache_layer=1)
    assert log == ["rms_norm", "matmul", "rotary", "forward", "crisp_cache_append", "quantize", "matmul"]


@pytest.mark.parametrize("tokens,hq,hkv", [(1024, HQ, HKV), (299, HQ, HKV), (301, HQ, HKV), (300, 32, 8), (300, HQ, 1), (300, 2, 2)])
def test_prompt_refuses_a_layer_of_another_size(log, block, tokens, hq, hkv):
    """The attention takes its sizes from the layer, and would read past the ends of shorter tensors."""
    with pytest.raises(ValueError):
        block.prompt(states(300), make_layer(log, tokens, hq, hkv))
    assert log == []


def test_prompt_refuses_a_layer_elsewhere(log, block):
    layer = make_layer(log, 300)
    layer.o = types.SimpleNamespace(device=torch.device("cuda", 1))
    with pytest.raises(ValueError):
        block.prompt(states(300), layer)
    with pytest.raises(ValueError):
        block.prompt(states(300)[0], make_layer(log, 300))
    assert log == []


@pytest.mark.parametrize("kw", [dict(seq_ids=None), dict(seq_ids=ids(0, 1)), dict(seq_ids=ids(0).long()), dict(seq_ids=ids(0), heads=1),
                                dict(seq_ids=ids(0), heads=8), dict(seq_ids=ids(0), cache_layer=2), dict(seq_ids=ids(0), cache_layer=-1),
                                dict(seq_ids=ids(0), device=torch.device("cuda", 1))])
def test_prompt_refuses_what_the_cache_would(log, block, kw):
    cache = make_cache(log, kw.get("heads", HKV), device=kw.get("device", CPU))
    with pytest.raises((ValueError, crisp.CrispError)):
        block.prompt(states(300), make_layer(log, 300), cache=cache, seq_ids=kw["seq_ids"], cache_layer=kw.get("cache_layer", 0))
    assert log == []


# ------------------------------------------------------------------------------------------------ a layer on another device
class Cuda:
    """Two devices, of which device 0 is current; the current streams have the handles 100 and 101."""

    def __init__(self, monkeypatch):
        self.now = 0
        cuda = self

        class Guard:
            def __init__(self, device):
                self.to = device if isinstance(device, int) else device.index

            def __enter__(self):
                self.back, cuda.now = cuda.now, self.to

            def __exit__(self, *args):
                cuda.now = self.back

        def current_stream(device=None):
            index = cuda.now if device is None else torch.device(device).index
            return types.SimpleNamespace(cuda_stream=100 + index)

        monkeypatch.setattr(torch.cuda, "device", Guard)
        monkeypatch.setattr(torch.cuda, "current_stream", current_stream)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: cuda.now)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index, raising=False)


@pytest.mark.parametrize("stream,handle", [(None, 101), (7, 7), (types.SimpleNamespace(cuda_stream=9), 9)])
def test_a_layer_s_calls_run_on_its_device(monkeypatch, stream, handle):
    """Whatever device is current, a layer's own is during its calls, and their stream is its current one if none is given."""
    cuda, given = Cuda(monkeypatch), []

    class Lib:
        def __getattr__(self, name):
            return lambda *args: given.append((name, cuda.now, args[-1])) or B.OK

    monkeypatch.setattr(B, "load", lambda: Lib())
    layer = object.__new__(crisp.CrispLayer)
    layer.p = crisp.make_params(300, HQ, HKV)
    for name in ("c_struct", "pattern", "p_v", "p_s", "row_ptr", "col_idx", "nnz", "lse"):
        setattr(layer, name, None)
    layer.route_ws = layer.select_ws = layer.prefill_ws = torch.zeros(256, dtype=torch.uint8)
    layer.capacity = 1
    layer.o = types.SimpleNamespace(device=torch.device("cuda", 1), data_ptr=lambda: 0)
    q = torch.zeros(1)
    layer.forward(q, q, q, stream=stream)
    layer.route(q, q, stream)
    layer.select(q, q, stream)
    layer.sparse_prefill(q, q, q, stream)
    layer.dense_prefill(q, q, q, stream)
    layer.poll(stream)
    assert [name for name, _, _ in given] == ["crisp_forward", "crisp_route", "crisp_select", "crisp_sparse_prefill",
                                              "crisp_dense_prefill"] + 3 * ["crisp_poll_device_status"]
    assert all(device == 1 and at == handle for _, device, at in given)
    assert cuda.now == 0


# ------------------------------------------------------------------------------------------------ an answer
def test_answer_calls(log, block):
    parts = ["rms_norm", "matmul", "rotary"], ["crisp_cache_append", "crisp_cache_attention", "quantize", "matmul"]
    first, later = parts[0] + ["crisp_cache_reserve"] + parts[1], parts[0] + parts[1]
    for kw, tokens, want in ((dict(), 3, first), (dict(cache_layer=1), 3, later), (dict(max_new=1), 3, first),
                             (dict(n_new=ids(2, 2, 2)), 6, first), (dict(n_new=ids(2, 2, 2), max_new=2), 6, first),
                             (dict(cu_tokens=ids(0, 1, 5, 5), n_new=ids(1, 4, 0)), 5, first), (dict(cache_layer=1), 6, later)):
        log.clear()
        block.answer(states(tokens), None, make_cache(log), ids(0, 4, 2), **kw)
        assert log == want, kw


@pytest.mark.parametrize("tokens,kw", [
    (3, dict(heads=1)), (3, dict(heads=8)),                                               # another number of K/V heads
    (3, dict(device=torch.device("cuda", 1))),
    (3, dict(cu_tokens=ids(0, 1, 2))), (3, dict(cu_tokens=ids(0, 1, 2, 3).long())),       # lists of the wrong length or type
    (3, dict(cu_tokens=ids(0, 0, 1, 1, 2, 2, 3, 3)[::2])), (3, dict(n_new=ids(1))), (3, dict(n_new=ids(1, 1, 1).float())),
    (3, dict(seq_ids=ids(0, 1, 2).long())), (3, dict(seq_ids=ids(0, 1, 2)[None])),
    (4, dict(n_new=ids(2, 1, 1))), (6, dict()), (0, dict()),                              # tokens that the sequences do not share out
    (6, dict(n_new=ids(2, 2, 2), max_new=1)), (3, dict(max_new=-1)), (3, dict(max_new=1 << 31)), (3, dict(max_new=1.0)),
    (3, dict(cache_layer=2)), (3, dict(cache_layer=-1)), (3, dict(cache_layer=0.0)),
    (1025, dict(seq_ids=torch.zeros(1025, dtype=torch.int32)))])
def test_a_refused_answer_leaves_the_sequences(log, block, tokens, kw):
    kw = dict(kw)
    cache = make_cache(log, kw.pop("heads", HKV), device=kw.pop("device", CPU))
    with pytest.raises((ValueError, TypeError, crisp.CrispError)):
        block.answer(states(tokens), None, cache, kw.pop("seq_ids", ids(0, 1, 2)), **kw)
    assert log == []


def test_answer_refuses_groups_that_attention_refuses(log):
    block = crisp.CrispAttention(linear((17 + 2) * 128, HIDDEN), linear(HIDDEN, 17 * 128), crisp.CrispRotary(1e4), 17, 1)
    with pytest.raises(crisp.CrispError):
        block.answer(states(1), None, make_cache(log, heads=1), ids(0))
    block = crisp.CrispAttention(linear((3 + 4) * 128, HIDDEN), linear(HIDDEN, 3 * 128), crisp.CrispRotary(1e4), 3, 2)
    with pytest.raises(crisp.CrispError):
        block.answer(states(1), None, make_cache(log, heads=2), ids(0))
    assert log == []


def test_prompt_refuses_a_cache_elsewhere(log, block):
    cache = make_cache(log)
    cache.device = torch.device("cuda", 1)
    cache._check = lambda *args: None      # its lists are there too
    with pytest.raises(ValueError):
        block.prompt(states(300), make_layer(log, 300), cache=cache, seq_ids=ids(0))
    assert log == []
