"""CrispAttention: norm, products, rotary positions and attention of a layer, from hidden states to hidden states, for prompts and
answers; and how its calls behave on streams, in graphs and beside one another."""
import numpy as np
import pytest
import torch

import paper_2609_01925_b200 as crisp
from tests import projection_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
HQ, HKV, HIDDEN = 4, 1, 512


def weights(n_out, n_in, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n_out, n_in, generator=g) * n_in ** -0.5).bfloat16()


def hidden(n, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, HIDDEN, generator=g) * size).bfloat16()


def make_block(seed=0, **rotary):
    w_qkv, w_o = weights((HQ + 2 * HKV) * 128, HIDDEN, seed), weights(HIDDEN, HQ * 128, seed + 1)
    w_norm = (1 + 0.1 * hidden(1, seed + 2)[0].float()).bfloat16()
    block = crisp.CrispAttention(crisp.CrispLinear.from_weight(w_qkv.to(DEV)), crisp.CrispLinear.from_weight(w_o.to(DEV)),
                                 crisp.CrispRotary(10000.0, **rotary), HQ, HKV, norm_weight=w_norm.to(DEV))
    return block, w_qkv, w_o, w_norm


def make_layer(n, seq=None):
    p = crisp.make_params(n, HQ, HKV, sink_tokens=4, local_tokens=min(128, n))
    return crisp.CrispLayer(p)


def f64(t):
    return t.detach().cpu().double().numpy()


def reference(x, residual, w_qkv, w_o, w_norm, freq):
    """The layer in float64 from the weights as they are held (8 bits), rounding where the layer stores 16 or 8 bits."""
    y, h = ref.norm(f64(x), None if residual is None else f64(residual), f64(w_norm), 1e-5)
    a = ref.values(*ref.quantize(y))
    qkv = ref.bf16(a @ ref.values(*ref.quantize(f64(w_qkv))).T).reshape(len(y), HQ + 2 * HKV, 128)
    turned = ref.bf16(ref.rotate(qkv[:, :HQ + HKV], range(len(y)), freq, "half"))
    q, k, v = turned[:, :HQ], turned[:, HQ:], qkv[:, HQ + HKV:]
    o = np.zeros_like(q)
    mask = np.tril(np.ones((len(y), len(y)), bool))
    for head in range(HQ):
        s = q[:, head] @ k[:, head * HKV // HQ].T / np.sqrt(128.0)
        s = np.where(mask, s, -np.inf)
        p = np.exp(s - s.max(1, keepdims=True))
        o[:, head] = p / p.sum(1, keepdims=True) @ v[:, head * HKV // HQ]
    out = ref.values(*ref.quantize(ref.bf16(o).reshape(len(y), -1))) @ ref.values(*ref.quantize(f64(w_o))).T
    return q, k, v, o, out, h


def rel(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("n", [100, 300, 777])
def test_prompt_against_float64(n):
    """Dense (below two blocks, or by the gate) a prompt is the formula's.  Values differ where a rounding of the norm's output or
    of attention's falls the other way: one e4m3 step (2^-3) of few elements; 16-bit roundings are 2^-8 of each."""
    block, w_qkv, w_o, w_norm = make_block()
    x, r = hidden(n, 5), hidden(n, 6, 2.0)
    q0, k0, v0, o0, out0, h0 = reference(x, r, w_qkv, w_o, w_norm, ref.frequencies(128, 10000.0))
    q, k, v, h = block.project(x.to(DEV), r.to(DEV))
    np.testing.assert_array_equal(f64(h), h0)
    for got, want in ((q, q0), (k, k0), (v, v0)):
        assert rel(f64(got), want) <= 2.0 ** -8
    out, h = block.prompt(x.to(DEV), make_layer(n), r.to(DEV), dense_below_tokens=1 << 20)
    block.poll()
    np.testing.assert_array_equal(f64(h), h0)
    # attention's output is rounded to e4m3 (half a step 2^-4 at most, relative): an element whose rounding falls the other way is a
    # whole step off; P in 8 bits of mantissa and O in 16 put that many elements near a border: 2^-8 / 2^-3 of them
    assert rel(f64(out), out0) <= 2.0 ** -8 + 2.0 ** -3 * np.sqrt(2.0 ** -5)


def test_prompt_is_its_calls():
    """prompt() gives, bit for bit, what the single calls give."""
    n = 1024
    block, *_ = make_block(3)
    x = hidden(n, 7).to(DEV)
    layer = make_layer(n)
    out, h = block.prompt(x, layer)
    assert h is None
    codes, scales, _ = crisp.rms_norm_quantize(x, block.norm_weight, eps=block.eps)
    q, k, v = block.rotary.split(block.qkv(codes, scales), HQ, HKV)
    o = make_layer(n).forward(q, k, v)
    again = block.out(*crisp.quantize(o.view(n, HQ * 128)))
    layer.poll()
    block.poll()
    assert torch.equal(out, again)


def test_answer_continues_a_prompt():
    """A prompt is stored and answered token by token; the answers agree with those of one longer prompt, within the cache's
    8 bits (e4m3: half a step 2^-4 of an element of K and V, so that much of o; measured against the size of the outputs)."""
    n, more = 384, 5
    block, *_ = make_block(4, layout="interleaved", rotary_dim=64)
    x, r = hidden(n + more, 8).to(DEV), hidden(n + more, 9).to(DEV)
    whole, _ = block.prompt(x, make_layer(n + more), r, dense_below_tokens=1 << 20)
    cache = crisp.CrispCache.allocate(16, HKV, 2, 8, fmt="e4m3")
    ids = torch.ones(1, dtype=torch.int32, device=DEV)
    first, _ = block.prompt(x[:n], make_layer(n), r[:n], cache=cache, seq_ids=ids, dense_below_tokens=1 << 20)
    assert torch.equal(first, whole[:n])
    got = []
    for t in range(n, n + more):
        position = torch.tensor([t], dtype=torch.int32, device=DEV)
        out, h = block.answer(x[t:t + 1], position, cache, ids, r[t:t + 1])
        got.append(out)
    cache.poll()
    block.poll()
    assert int(cache.seq_lens[1]) == n + more
    assert rel(f64(torch.cat(got)), f64(whole[n:])) <= 2.0 ** -4 + 2.0 ** -4   # the cache's rounding, and the other way at the output's


def test_answers_of_several_layers_and_sequences():
    """Two layers, three sequences at their own positions: the same as each sequence alone."""
    layers, lens = 2, [130, 1, 257]
    blocks = [make_block(10 + i)[0] for i in range(layers)]
    steps = [hidden(3, 20 + i).to(DEV) for i in range(layers)]

    def run(which):
        cache = crisp.CrispCache.allocate(16, HKV, 3, 8, n_layers=layers, fmt="int8")
        ids = torch.tensor(which, dtype=torch.int32, device=DEV)
        total = sum(lens[i] for i in which)
        cu = torch.tensor(np.concatenate([[0], np.cumsum([lens[i] for i in which])]), dtype=torch.int32, device=DEV)
        new = torch.tensor([lens[i] for i in which], dtype=torch.int32, device=DEV)
        begin = torch.cat([hidden(lens[i], 30 + i) for i in which]).to(DEV)
        positions = torch.cat([torch.arange(lens[i]) for i in which]).int().to(DEV)
        assert begin.shape[0] == total
        for layer, block in enumerate(blocks):
            block.answer(begin, positions, cache, ids, cu_tokens=cu, n_new=new, cache_layer=layer)
        outs = []
        for layer, block in enumerate(blocks):
            x = steps[layer][which].contiguous()
            outs.append(block.answer(x, torch.tensor([lens[i] for i in which], dtype=torch.int32, device=DEV), cache, ids,
                                     cache_layer=layer)[0])
        cache.poll()
        return [f64(o) for o in outs]

    together = run([0, 1, 2])
    for i in range(3):
        alone = run([i])
        for a, b in zip(alone, together):
            # sums in another order (fp32), then a rounding to 16 bits and one to 8 that may fall the other way
            assert rel(a[0], b[i]) <= 2.0 ** -4


# ------------------------------------------------------------------------------------------------ streams, graphs, neighbours
def answer_step(block, x, positions, cache, ids):
    return block.answer(x, positions, cache, ids)[0]


def test_captured_step_replays():
    """An answering step in a CUDA graph: replayed on new inputs it gives what the eager calls give."""
    block, *_ = make_block(40)

    def start():
        cache = crisp.CrispCache.allocate(16, HKV, 2, 8)
        ids = torch.zeros(1, dtype=torch.int32, device=DEV)
        begin = hidden(200, 41).to(DEV)
        block.answer(begin, torch.arange(200, dtype=torch.int32, device=DEV), cache, ids,
                     n_new=torch.tensor([200], dtype=torch.int32, device=DEV))
        return cache, ids

    xs = [hidden(1, 50 + i).to(DEV) for i in range(4)]
    cache, ids = start()
    eager = [answer_step(block, x, torch.tensor([200 + i], dtype=torch.int32, device=DEV), cache, ids) for i, x in enumerate(xs)]
    cache2, ids2 = start()
    x, position = xs[0].clone(), torch.tensor([200], dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = answer_step(block, x, position, cache2, ids2)
    for i in range(4):
        x.copy_(xs[i])
        position.fill_(200 + i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i]), i
    cache2.poll()
    block.poll()


def test_first_calls_of_a_process_may_be_captured():
    """Nothing that a call does for the first time gets in the way of a capture."""
    import subprocess
    import sys
    code = """
import torch, paper_2609_01925_b200 as crisp
x = torch.randn(400, 512, device="cuda").bfloat16(); w = torch.randn(1024, 512, device="cuda").bfloat16()
rot = crisp.CrispRotary(1e4); torch.cuda.synchronize()
s = torch.cuda.Stream()
ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
g = torch.cuda.CUDAGraph()
lin = crisp.CrispLinear(torch.empty(1024, 512, device="cuda").to(torch.float8_e4m3fn), torch.empty(1024, 4, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu))
torch.cuda.synchronize()
def step(x):
    c, sc, _ = crisp.rms_norm_quantize(x)
    wc, ws = crisp.quantize(w)
    lin.codes.copy_(wc.view(torch.uint8).view(torch.float8_e4m3fn)); lin.scales.view(torch.uint8).copy_(ws.view(torch.uint8))
    return rot.split(lin(c, sc), 4, 2), rot.split(lin(c[:5].contiguous(), sc[:5].contiguous()), 4, 2)
with torch.cuda.graph(g):
    out = step(x)
g.replay(); torch.cuda.synchronize()
want = step(x); torch.cuda.synchronize(); lin.poll()
assert all(torch.equal(a, b) for p, q in zip(out, want) for a, b in zip(p, q))
print("ok")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=root)
    assert done.returncode == 0 and "ok" in done.stdout, done.stderr[-2000:]


def test_two_graphs_share_a_linear():
    """Two captured products of one CrispLinear, replayed at the same time on two streams."""
    w = weights(1024, 2048, 60)
    lin = crisp.CrispLinear.from_weight(w.to(DEV))
    sets = [crisp.quantize(torch.randn(m, 2048, device=DEV).bfloat16()) for m in (3, 200)]
    want = [lin(*s) for s in sets]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(lin(*s))
        graphs.append(g)
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    lin.poll()
    for a, b in zip(outs, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("handle", [False, True])
def test_calls_on_a_given_stream(handle):
    """Inputs dropped right behind the calls, work on another stream than the current one: the same results."""
    block, *_ = make_block(70)
    xs = [hidden(257, 71 + i).to(DEV) for i in range(6)]
    want = [block.project(x) for x in xs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    stream = side.cuda_stream if handle else side
    got = []
    for x in xs:
        torch.cuda._sleep(200000)
        y = x.clone()
        side.wait_stream(torch.cuda.current_stream())
        got.append(block.project(y, stream=stream))
        del y
        torch.empty(257, HIDDEN, dtype=torch.bfloat16, device=DEV).fill_(float("nan"))   # takes memory that was freed too early
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(s, t) for s, t in zip(a[:3], b[:3]))


@pytest.mark.parametrize("given", [False, True])
def test_inputs_of_another_stream_may_be_dropped(given):
    """Tensors of the default stream, used by calls on a side stream (the current one, or given) that run late, and dropped right
    behind them: their memory is not handed out before."""
    block, *_ = make_block(170)
    xs = [hidden(257, 171 + i).to(DEV) for i in range(4)]
    residual, positions = hidden(257, 180).to(DEV), torch.arange(257, dtype=torch.int32, device=DEV)
    want = [block.project(x, residual, positions) for x in xs]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for x in xs:
        inputs = [t.clone() for t in (x, residual, positions)]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(2000000)
            got.append(block.project(*inputs, stream=side if given else None))
        del inputs
        for t in (x, residual, positions):
            torch.empty_like(t).fill_(7)     # takes memory that was freed too early
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_default_stream_as_zero():
    block, *_ = make_block(80)
    x = hidden(33, 81).to(DEV)
    want = block.project(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = block.project(x, stream=0)
    torch.cuda.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(got[:3], want[:3]))


def test_weights_written_just_before():
    """Weights converted by the call right before the product: nothing of them is read too early."""
    x = crisp.quantize(torch.randn(5, 4096, device=DEV).bfloat16())
    w = [torch.randn(6144, 4096, device=DEV).bfloat16() for _ in range(2)]
    want = [crisp.CrispLinear.from_weight(t)(*x) for t in w]
    torch.cuda.synchronize()
    codes, scales = crisp.quantize(w[0])
    lin = crisp.CrispLinear(codes, scales)
    for i in range(6):
        from paper_2609_01925_b200 import binding as B
        B.check(B.crisp_quantize(w[i % 2], codes, scales), "crisp_quantize")
        assert torch.equal(lin(*x), want[i % 2]), i


def test_block_refusals():
    block, *_ = make_block(90)
    with pytest.raises(ValueError):
        crisp.CrispAttention(block.out, block.qkv, block.rotary, HQ, HKV)
    with pytest.raises(ValueError):
        block.project(hidden(3, 1).to(DEV)[:, :256].contiguous())
    with pytest.raises(ValueError):
        block.project(hidden(3, 1).to(DEV), positions=torch.zeros(2, dtype=torch.int32, device=DEV))


def test_refused_calls_leave_the_cache():
    """A prompt or an answer that does not fit its layer or its cache raises, and no sequence has grown."""
    block, *_ = make_block(95)
    cache = crisp.CrispCache.allocate(8, HKV, 2, 4)
    other = crisp.CrispCache.allocate(8, 2 * HKV, 2, 4)
    ids = torch.zeros(1, dtype=torch.int32, device=DEV)
    first, _ = block.prompt(hidden(130, 96).to(DEV), make_layer(130), cache=cache, seq_ids=ids, dense_below_tokens=1 << 20)
    x, at = hidden(1, 97).to(DEV), torch.tensor([130], dtype=torch.int32, device=DEV)
    wide = crisp.CrispLayer(crisp.make_params(130, 2 * HQ, HKV, sink_tokens=4))
    for bad in (lambda: block.prompt(hidden(10, 98).to(DEV), make_layer(130)), lambda: block.prompt(hidden(131, 98).to(DEV), make_layer(130)),
                lambda: block.prompt(hidden(130, 98).to(DEV), wide),
                lambda: block.prompt(hidden(130, 98).to(DEV), make_layer(130), cache=other, seq_ids=ids),
                lambda: block.answer(x, at, other, ids), lambda: block.answer(x, at, cache, ids, cu_tokens=ids),
                lambda: block.answer(x, at, cache, ids, max_new=0), lambda: block.answer(x, at, cache, ids, n_new=ids.long()),
                lambda: block.answer(x, at.long(), cache, ids), lambda: block.answer(x, at, cache, ids, cache_layer=1),
                lambda: block.answer(torch.cat([x, x]), torch.cat([at, at + 1]), cache, ids)):
        with pytest.raises((ValueError, crisp.CrispError)):
            bad()
    torch.cuda.synchronize()
    assert cache.seq_lens.tolist() == [130, 0] and other.seq_lens.tolist() == [0, 0]
    block.answer(x, at, cache, ids, max_new=1)
    cache.poll()
    other.poll()
    block.poll()
    assert cache.seq_lens.tolist() == [131, 0]
