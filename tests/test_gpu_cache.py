"""The paged 8-bit cache on the GPU against a plain cache in float64 (cache_reference.py): the quantising write and the
page operations are exact and compared for equality; attention within bounds derived from its roundings."""
import numpy as np
import pytest
import torch

import paper_2609_01925_b200 as crisp
from paper_2609_01925_b200 import binding as B
from tests import cache_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"


def i32(x):
    return torch.tensor([int(v) for v in x], dtype=torch.int32, device=DEV)


def tokens(n, heads, seed, spread=0.0):
    """bf16 [n, heads, 128]; with `spread` the tokens' magnitudes differ by powers of two up to 2^spread."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, heads, 128, generator=g)
    if spread:
        x = x * torch.exp2(torch.rand(n, heads, 1, generator=g) * spread - spread / 2)
    return x.bfloat16()


class Both:
    """A cache on the GPU and its reference, driven by the same calls."""

    def __init__(self, fmt, heads, pages, max_seqs, max_pages, layers=1, garbage=True):
        self.gpu = crisp.CrispCache.allocate(pages, heads, max_seqs, max_pages, n_layers=layers, fmt=fmt)
        if garbage:   # what no token has been written to holds NaN codes and NaN scales
            for t in (self.gpu.k_codes, self.gpu.v_codes):
                t.fill_(0xff)
            for t in (self.gpu.k_scale, self.gpu.v_scale):
                t.fill_(float("nan"))
        self.ref = ref.RefCache(layers, pages, heads, max_seqs, max_pages, fmt)

    def grow(self, ids, n_new, seed, spread=0.0, layers=None):
        """reserve, and append of random tokens to every layer (or the given ones)."""
        heads = self.ref.heads
        cu = np.concatenate([[0], np.cumsum(n_new)]).tolist()
        self.gpu.reserve(i32(ids), i32(n_new))
        self.ref.reserve(ids, n_new)
        for layer in range(self.ref.layers) if layers is None else layers:
            k, v = (tokens(cu[-1], heads, seed + 100003 * (2 * layer + j), spread) for j in range(2))
            self.gpu.append(k.to(DEV), v.to(DEV), i32(ids), i32(cu), layer=layer)
            self.ref.append(k.double().numpy(), v.double().numpy(), ids, cu, layer)

    def check_tables(self):
        self.gpu.poll()
        assert np.array_equal(self.gpu.seq_lens.cpu().numpy(), self.ref.lens)
        assert np.array_equal(self.gpu.page_refs.cpu().numpy(), self.ref.refs)
        assert np.array_equal(self.gpu.page_table.cpu().numpy(), self.ref.table)

    def check_contents(self):
        """Every stored token's codes and every used block's scale are those of the reference."""
        for name, codes, scale in (("k", self.gpu.k_codes, self.gpu.k_scale), ("v", self.gpu.v_codes, self.gpu.v_scale)):
            codes, scale = codes.cpu().numpy(), scale.cpu().numpy()
            for s in range(self.ref.max_seqs):
                n = self.ref.lens[s]
                for j in range(ref.pages_of(n)):
                    p, rows = self.ref.table[s, j], min(128, n - 128 * j)
                    got = ref.values(codes[:, p, :, :rows], self.ref.fmt)
                    want = ref.values(self.ref.codes[name][:, p, :, :rows], self.ref.fmt)
                    np.testing.assert_array_equal(got, want)
                    np.testing.assert_array_equal(scale[:, p], 2.0 ** self.ref.exps[name][:, p])

    def check_attention(self, hq, ids, n_new, seed, layer=0, q=None, cu=None, **kw):
        if cu is None:
            cu = np.concatenate([[0], np.cumsum(n_new)]).tolist()
        if q is None:
            q = tokens(cu[-1], hq, seed)
        lse = torch.full((hq, q.shape[0]), 7.0, device=DEV)
        o = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        out = self.gpu.attention(q.to(DEV), i32(ids), i32(cu), max_new=max(n_new), layer=layer, o=o, lse=lse, **kw)
        assert out is o
        self.gpu.poll()
        rows = max(n_new) * hq // self.ref.heads
        want = self.ref.attention(q.double().numpy(), ids, cu, layer)
        check_rows(o, lse, want, rows)
        return o, lse


def check_rows(o, lse, reference, rows, untouched=7.0):
    want, want_lse, slack, dots = reference
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    none = np.isnan(want)
    assert (o[none] == untouched).all() and (lse[np.isnan(want_lse)] == untouched).all()
    # weights are rounded to fp16 (2^-11) by the kernel for few rows, to bf16 (2^-8) by the one for many
    tol = ref.tolerance(want, slack, 2.0 ** -11 if rows <= 24 else 2.0 ** -8, 64)
    bad = ~none & ~(np.abs(o - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], np.nanmax(np.abs(o - want) / tol))
    fin = np.isfinite(want_lse)
    assert np.array_equal(lse == -np.inf, want_lse == -np.inf)
    assert (np.abs(lse[fin] - want_lse[fin]) <= ref.lse_tolerance(want_lse[fin], dots[fin], 64)).all()


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("spread", [0.0, 12.0, 60.0])
def test_append_in_pieces_equals_the_definition(fmt, spread):
    """Pieces of one token, across page borders, of whole pages, from sequences in any order; scales that grow."""
    both = Both(fmt, heads=3, pages=24, max_seqs=5, max_pages=6)
    seed = 0
    for ids, n_new in (([2, 0, 4], [1, 127, 130]), ([0, 2], [1, 1]), ([4, 2, 0], [126, 255, 2]), ([1], [300]),
                       ([0, 1, 2, 4], [1, 1, 1, 1]), ([3, 1], [0, 1]), ([-1, 3, -1], [0, 5, 0])):
        both.grow(ids, n_new, seed, spread)
        seed += 2
        both.check_tables()
        both.check_contents()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_of_extreme_values(fmt):
    """Zeros, infinities, NaN, the largest and the smallest bf16 numbers, exact ties and scale borders."""
    both = Both(fmt, heads=2, pages=8, max_seqs=2, max_pages=4)
    k, v = tokens(200, 2, 1), tokens(200, 2, 2)
    top = torch.finfo(torch.bfloat16).max
    k[0, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), -0.0])
    k[1, 1] = 0
    k[5, 0, 7] = 448 * 2.0 ** 3             # exactly the border of e = 3 (e4m3)
    v[:128, 0] = 0                          # a block of zeros
    v[128:, 0] *= 2.0 ** -130               # subnormal values
    v[3, 1, 5] = top
    k[130:, 1] = torch.linspace(-508, 508, 70)[:, None].bfloat16().expand(70, 128)   # ties on the int8 grid
    both.gpu.reserve(i32([1]), i32([200]))
    both.ref.reserve([1], [200])
    both.gpu.append(k.to(DEV), v.to(DEV), i32([1]))
    both.ref.append(k.double().numpy(), v.double().numpy(), [1], [0, 200])
    both.check_tables()
    both.check_contents()


def test_append_writes_only_its_layer_and_its_rows():
    both = Both("e4m3", heads=2, pages=6, max_seqs=3, max_pages=2, layers=3)
    both.grow([1, 0], [100, 20], 5, layers=[1])
    got = both.gpu.k_codes.cpu().numpy()
    assert (got[[0, 2]] == 0xff).all()
    assert (got[1, both.ref.table[1, 0], :, 100:] == 0xff).all() and (got[1, both.ref.table[0, 0], :, 20:] == 0xff).all()
    assert (got[1, 2:] == 0xff).all()


# ------------------------------------------------------------------------------------------------ attention
SHAPES = [(4, 1), (8, 2), (7, 1), (2, 2), (16, 1), (6, 2)]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hkv", SHAPES)
def test_one_token_at_many_lengths(fmt, hq, hkv):
    lens = [1, 2, 31, 32, 33, 127, 128, 129, 300, 1000]
    both = Both(fmt, hkv, pages=40, max_seqs=len(lens), max_pages=8)
    both.grow(list(range(len(lens))), lens, 11, spread=2.0)
    ids = [3, 9, 0, 1, 7, 2, 8, 4, 5, 6]
    both.check_attention(hq, ids, [1] * len(ids), 12)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hkv", SHAPES)
@pytest.mark.parametrize("new", [[2, 1, 3, 2], [5, 1, 0, 4], [9, 30, 16, 1]])
def test_several_new_tokens(fmt, hq, hkv, new):
    lens = [2, 130, 300, 517]
    both = Both(fmt, hkv, pages=16, max_seqs=4, max_pages=6)
    both.grow([0, 1, 2, 3], [max(n, m) for n, m in zip(lens, new)], 21)
    both.check_attention(hq, [0, 1, 2, 3], new, 22)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hkv,new,lens", [
    (4, 1, [200], [200]),                      # a whole prompt: nothing is cached before it
    (4, 1, [64, 65, 1, 128], [700, 65, 3, 1000]),
    (7, 1, [36, 37, 150], [513, 90, 150]),     # groups of seven: 36 tokens (252 rows) to a pair of tiles
    (2, 2, [256, 300], [257, 900]),
    (16, 1, [16, 17, 100], [16, 300, 129]),
    (6, 2, [90, 85], [640, 85]),
    (1, 1, [128, 129, 511], [128, 400, 511]),
])
def test_long_pieces(fmt, hq, hkv, new, lens):
    both = Both(fmt, hkv, pages=30, max_seqs=len(lens), max_pages=9)
    both.grow(list(range(len(lens))), lens, 25, spread=2.0)
    ids = list(range(len(lens)))[::-1]
    both.check_attention(hq, ids, [new[i] for i in ids], 26)


def test_long_piece_over_a_long_cache_is_cut_and_joined():
    both = Both("e4m3", 1, pages=170, max_seqs=2, max_pages=160)
    both.grow([1, 0], [20000, 300], 45)
    both.check_attention(4, [1], [40], 46)
    both.check_attention(4, [0, 1], [70, 3], 47)


@pytest.mark.parametrize("new", [1, 3, 9])
def test_an_empty_cache_answers_zeros(new):
    """Nothing has been written anywhere: codes and scales are NaN."""
    both = Both("e4m3", 1, pages=2, max_seqs=2, max_pages=2)
    o, lse = both.check_attention(4, [1, 0], [new, new], 33)
    assert (o == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("new", [1, 3, 9])
def test_rows_that_see_nothing_and_padding(new):
    """Empty sequences, more queries than keys, padding entries, tokens behind the last item: zeros or untouched."""
    both = Both("e4m3", 2, pages=8, max_seqs=5, max_pages=3)
    both.grow([1, 3], [2, 200], 31)
    ids = [0, 1, -1, 3, 4]
    cu = [0, new, new + 3, new + 4, new + 5, new + 6]   # the pieces of one call go to one kernel, by the longest
    q = tokens(cu[-1] + 2, 8, 32)
    o, lse = both.check_attention(8, ids, [max(new, 3)], 0, q=q, cu=cu)
    assert (o[:new] == 0).all() and (lse[:, :new] == -float("inf")).all()
    assert (o[new] == 0).all()           # the first of three queries over two keys
    assert (o[-2:] == 7).all() and (o[new + 3] == 7).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_long_sequences_are_cut_and_joined(fmt):
    """A single long sequence is spread over all CTAs (two levels of joining), beside short ones."""
    both = Both(fmt, 1, pages=420, max_seqs=3, max_pages=400)
    both.grow([1, 0, 2], [50000, 5, 777], 41)
    both.check_attention(4, [1], [1], 42)
    both.check_attention(4, [0, 1, 2], [1, 1, 1], 43)
    both.check_attention(4, [1, 2], [5, 2], 44)


def test_very_different_scales_between_pages():
    """Pages whose scales differ by 2^100 in V and by 2^20 in K."""
    both = Both("e4m3", 1, pages=8, max_seqs=1, max_pages=6)
    for i, (ek, ev) in enumerate([(0, 0), (-10, 60), (10, -40), (0, -126)]):
        k, v = tokens(128, 1, 50 + 2 * i) * 2.0 ** ek, tokens(128, 1, 51 + 2 * i) * 2.0 ** ev
        both.gpu.reserve(i32([0]), i32([128]))
        both.ref.reserve([0], [128])
        both.gpu.append(k.to(DEV), v.to(DEV), i32([0]))
        both.ref.append(k.double().numpy(), v.double().numpy(), [0], [0, 128])
    for new in (2, 20):
        q = tokens(new, 4, 60)
        q[0] *= 2.0 ** -120
        q[1, :, ::3] *= 2.0 ** -9        # elements far below the row's largest
        both.check_attention(4, [0], [new], 0, q=q)


@pytest.mark.parametrize("new", [1, 3, 5, 20])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_sink_leaves_the_other_weights_their_bits(fmt, new):
    """The first token takes all weight but 2^-22 of it and has no value.  What is left comes from weights of 2^-18 to 2^-27 in
    its page, or from weights of about 2^-37 in a page whose values are 2^30 times larger."""
    for page2 in (0.0, 2.0 ** 30):
        both = Both(fmt, 1, pages=4, max_seqs=1, max_pages=4)
        k, v = tokens(256, 1, 801), tokens(256, 1, 802)
        k[0], v[0] = 15.5 / 128 ** 0.5, 0           # a logit of 15.5 with queries near (1, 1, ...)
        k[128:] -= 10 / 128 ** 0.5
        v[128:] *= page2
        v[160:] = 0                                 # the tokens that share a warp with the sink
        both.gpu.reserve(i32([0]), i32([256]))
        both.ref.reserve([0], [256])
        both.gpu.append(k.to(DEV), v.to(DEV), i32([0]))
        both.ref.append(k.double().numpy(), v.double().numpy(), [0], [0, 256])
        q = (1 + tokens(new, 4, 803) / 16).bfloat16()
        both.check_attention(4, [0], [new], 0, q=q)


@pytest.mark.parametrize("new", [2, 20])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_very_large_logits(fmt, sign, new):
    """Logits of 1e33, 1e10, 1e9 (between 0.9 and 1.4 times 2^30 in base 2) and 1e8: the keys come in a few exact sizes, mixed or
    a size for each half of a page, so the nearest ones share all weight."""
    for size in (torch.arange(300) % 7, torch.arange(300) // 64):
        k = (sign * (1 + size / 8) * 2.0 ** 40)[:, None, None].expand(300, 1, 128).bfloat16()
        v = tokens(300, 1, 805)
        both = Both(fmt, 1, pages=4, max_seqs=1, max_pages=4)
        both.gpu.reserve(i32([0]), i32([300]))
        both.ref.reserve([0], [300])
        both.gpu.append(k.contiguous().to(DEV), v.to(DEV), i32([0]))
        both.ref.append(k.double().numpy(), v.double().numpy(), [0], [0, 300])
        assert np.array_equal(both.ref.states("k", 0), k.double().numpy())       # exact in both formats
        for top in (2.0 ** 66, 2.0 ** -10, 1.75 * 2.0 ** -15, 2.0 ** -16):
            q = torch.full((new, 4, 128), top, dtype=torch.bfloat16)
            lse = torch.empty(4, new, device=DEV)
            o = both.gpu.attention(q.to(DEV), i32([0]), lse=lse)
            both.gpu.poll()
            want, want_lse, slack, dots = both.ref.attention(q.double().numpy(), [0], [0, new])
            # equal keys give equal logits and the others' weights are 0, so the logits' own error drops out of slack
            tol = ref.tolerance(want, slack / (1 + dots.T[:, :, None]), 2.0 ** -11 if new <= 6 else 2.0 ** -8, 64)
            assert (np.abs(o.double().cpu().numpy() - want) <= tol).all()
            assert (np.abs(lse.double().cpu().numpy() - want_lse) <= ref.lse_tolerance(want_lse, dots, 64)).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_very_large_values(fmt):
    """V up to 2^119: scales beyond 2^105, in both kernels."""
    both = Both(fmt, 1, pages=4, max_seqs=1, max_pages=4)
    for i, ev in enumerate((117, 105, 111)):
        n = 128 if i < 2 else 70
        k, v = tokens(n, 1, 63 + 2 * i), tokens(n, 1, 64 + 2 * i) * 2.0 ** ev
        both.gpu.reserve(i32([0]), i32([n]))
        both.ref.reserve([0], [n])
        both.gpu.append(k.to(DEV), v.to(DEV), i32([0]))
        both.ref.append(k.double().numpy(), v.double().numpy(), [0], [0, n])
    assert both.ref.exps["v"][0, :3, 0].min() > 95
    for new in (2, 20):
        both.check_attention(4, [0], [new], 69 + new)


@pytest.mark.parametrize("new", [2, 20])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_the_largest_value_is_hidden_like_any_other(fmt, new):
    """The last token's V is the largest bf16 number, whose nearest code stands for 2^128: the rows before do not see it."""
    both = Both(fmt, 1, pages=4, max_seqs=1, max_pages=4)
    k, v = tokens(148, 1, 65), tokens(148, 1, 66)
    v[128:147] *= 2.0 ** 112
    v[147] = torch.finfo(torch.bfloat16).max
    both.gpu.reserve(i32([0]), i32([148]))
    both.ref.reserve([0], [148])
    both.gpu.append(k.to(DEV), v.to(DEV), i32([0]))
    both.ref.append(k.double().numpy(), v.double().numpy(), [0], [0, 148])
    assert both.ref.states("v", 0)[147].max() == 2.0 ** 128
    q = tokens(new, 4, 67)
    lse = torch.full((4, new), 7.0, device=DEV)
    o = both.gpu.attention(q.to(DEV), i32([0]), lse=lse)
    both.gpu.poll()
    want, want_lse, slack, dots = both.ref.attention(q.double().numpy(), [0], [0, new])
    check_rows(o[:-1], lse[:, :-1], (want[:-1], want_lse[:, :-1], slack[:-1], dots[:, :-1]), 4 * new)


@pytest.mark.parametrize("new", [1, 5, 20])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_not_finite_queries_and_keys_reach_their_rows_only(fmt, new):
    """A row of Q with an infinity or NaN gives NaN in its own output; in e4m3 a NaN key reaches the rows that see it."""
    both = Both(fmt, 1, pages=8, max_seqs=2, max_pages=4)
    both.grow([0, 1], [300, 200], 61)
    q = tokens(2 * new, 4, 62)
    clean = both.gpu.attention(q.to(DEV), i32([0, 1]), max_new=new)
    q[0, 1, 5], q[new, 3, 7] = float("nan"), float("inf")
    o = both.gpu.attention(q.to(DEV), i32([0, 1]), max_new=new)
    bad = torch.zeros(2 * new, 4, dtype=torch.bool)
    bad[0, 1] = bad[new, 3] = True
    assert o[bad].isnan().all() and torch.equal(o[~bad], clean[~bad])
    if fmt == "e4m3":
        page = both.ref.table[0, 2]
        both.gpu.k_codes[0, page, 0, 300 - 256 - 1, 9] = 0x7f        # the last token: seen by the last query only
        o = both.gpu.attention(q.to(DEV), i32([0, 1]), max_new=new)
        bad[new - 1] = True
        assert o[bad].isnan().all() and torch.equal(o[~bad], clean[~bad])


def test_layers_and_scale_and_repeats():
    both = Both("int8", 2, pages=12, max_seqs=3, max_pages=4, layers=2)
    both.grow([0, 2], [300, 10], 71)
    both.check_attention(4, [2, 0, 0, 2], [1, 1, 1, 1], 72, layer=1)   # a sequence may be read twice
    both.check_attention(4, [2, 0, 0, 2], [1, 100, 9, 9], 74, layer=1)
    q = tokens(2, 4, 73)
    o = both.gpu.attention(q.to(DEV), i32([0, 2]), layer=1, softmax_scale=0.5)
    want, _, slack, _ = ref.attention(lambda s: (both.ref.states("k", s, 1), both.ref.states("v", s, 1)),
                                   q.double().numpy(), [0, 2], [0, 1, 2], 0.5)
    assert (np.abs(o.double().cpu().numpy() - want) <= ref.tolerance(want, slack, 2.0 ** -11, 64)).all()


@pytest.mark.parametrize("new", [2, 20])
@pytest.mark.parametrize("scale,eq", [(1.5e38, -124), (3e-38, 120), (1e-44, 126)])
def test_extreme_softmax_scales(scale, eq, new):
    """The largest and the smallest scales, over queries that bring the logits back to ordinary size."""
    both = Both("e4m3", 2, pages=8, max_seqs=1, max_pages=4)
    both.grow([0], [300], 75)
    q = (tokens(new, 4, 76) / 8).clamp(-1, 1) * 2.0 ** eq
    lse = torch.empty(4, new, device=DEV)
    o = both.gpu.attention(q.to(DEV), i32([0]), softmax_scale=scale, lse=lse)
    both.gpu.poll()
    scale = float(np.float32(scale))
    check_rows(o, lse, both.ref.attention(q.double().numpy(), [0], [0, new], scale=scale), 2 * new)


def test_same_call_same_bits_and_uniform_form():
    both = Both("e4m3", 2, pages=200, max_seqs=4, max_pages=100)
    both.grow([0, 1, 2], [9000, 300, 4000], 81)
    q = tokens(6, 8, 82).to(DEV)
    # (max_new picks the kernel, so the two forms are compared under the same bound)
    a = both.gpu.attention(q, i32([2, 0, 1]), i32([0, 2, 4, 6]), max_new=2)
    b = both.gpu.attention(q, i32([2, 0, 1]))
    c = both.gpu.attention(q, i32([2, 0, 1]))
    assert torch.equal(b, c) and torch.equal(a, b)
    q = tokens(150, 8, 83).to(DEV)
    a, b, c = (both.gpu.attention(q, i32([2, 0, 1]), cu) for cu in (i32([0, 50, 100, 150]), None, None))
    assert torch.equal(b, c) and torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ pages
def test_pages_random_walk():
    """Reserve, append, fork (shared and copied, whole and cut), free and compact in random order: tables equal, and
    contents of all that is stored equal."""
    rng = np.random.RandomState(3)
    both = Both("e4m3", heads=1, pages=60, max_seqs=8, max_pages=7, layers=2)
    for step in range(120):
        live = [s for s in range(8) if both.ref.lens[s] > 0]
        empty = [s for s in range(8) if both.ref.lens[s] == 0]
        op = rng.randint(5)
        try:
            if op <= 1:
                ids = rng.permutation(8)[:rng.randint(1, 5)].tolist()
                n = [int(rng.choice([1, 1, 7, 128, 200])) for _ in ids]
                if any(both.ref.lens[s] + m > 7 * 128 for s, m in zip(ids, n)):
                    continue
                both.ref._take(sum(ref.pages_of(both.ref.lens[s] + m) - ref.pages_of(both.ref.lens[s]) for s, m in zip(ids, n)))
                both.grow(ids, n, 1000 + 2 * step, spread=4.0)
            elif op == 2 and live and empty:
                dst = empty[:rng.randint(1, len(empty) + 1)]
                src = [int(rng.choice(live)) for _ in dst]
                n = [int(rng.randint(0, both.ref.lens[s] + 1)) for s in src] if rng.randint(2) else None
                share = bool(rng.randint(3))
                both.ref.fork(src, dst, n, share)
                both.gpu.fork(i32(src), i32(dst), None if n is None else i32(n), share)
            elif op == 3:
                ids = rng.permutation(8)[:rng.randint(1, 4)].tolist()
                ids = ids + ids[:1] + [-1]        # twice, and padding
                both.ref.free(ids)
                both.gpu.free(i32(ids))
            else:
                assert int(both.gpu.compact().item()) == both.ref.compact()
        except ref.Refused:
            continue
        both.check_tables()
    both.check_contents()


def test_calls_that_do_not_fit_change_nothing():
    both = Both("e4m3", heads=1, pages=4, max_seqs=4, max_pages=3)
    both.grow([0, 1], [130, 100], 91)
    before = [t.clone() for t in (both.gpu.page_table, both.gpu.seq_lens, both.gpu.page_refs, both.gpu.k_codes)]

    def refused(code, call, *args, **kw):
        call(*args, **kw)
        with pytest.raises(crisp.CrispError) as e:
            both.gpu.poll()
        assert e.value.status == code
        both.gpu.poll()
        for a, b in zip(before, (both.gpu.page_table, both.gpu.seq_lens, both.gpu.page_refs, both.gpu.k_codes)):
            assert torch.equal(a, b)

    refused(B.ERR_NO_PAGES, both.gpu.reserve, i32([2, 1]), i32([128, 29]))          # two pages, one free
    refused(B.ERR_NO_PAGES, both.gpu.reserve, i32([0]), i32([300]))                 # longer than a row
    refused(B.ERR_BAD_CACHE, both.gpu.reserve, i32([2, 2]), i32([1, 1]))            # twice
    refused(B.ERR_BAD_CACHE, both.gpu.reserve, i32([4]))                            # no such sequence
    refused(B.ERR_BAD_CACHE, both.gpu.reserve, i32([0]), i32([-1]))
    refused(B.ERR_NO_PAGES, both.gpu.fork, i32([0, 1]), i32([2, 3]))                # two copies, one free
    refused(B.ERR_BAD_CACHE, both.gpu.fork, i32([0]), i32([1]))                     # not empty
    refused(B.ERR_BAD_CACHE, both.gpu.fork, i32([0, 1]), i32([2, 2]))               # twice
    refused(B.ERR_BAD_CACHE, both.gpu.fork, i32([0]), i32([2]), i32([131]))         # longer than its source
    refused(B.ERR_BAD_CACHE, both.gpu.free, i32([9]))


def tensors(c):
    return (c.page_table, c.seq_lens, c.page_refs, c.k_codes, c.v_codes, c.k_scale, c.v_scale)


def raises_at_poll(c, code):
    with pytest.raises(crisp.CrispError) as e:
        c.poll()
    assert e.value.status == code
    c.poll()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_step_behind_a_refused_reserve_leaves_the_cache_as_it_was(fmt):
    """reserve (no page for one of its sequences), append of two layers, attention, without a poll between; then a page is
    freed and the same step succeeds."""
    both = Both(fmt, heads=2, pages=5, max_seqs=4, max_pages=3, layers=2)
    both.grow([0, 1, 2], [128, 130, 90], 701)
    both.grow([3], [5], 703)
    c = both.gpu
    before = [t.clone() for t in tensors(c)]
    k, v, q = (tokens(3, h, 705 + j).to(DEV) * 64 for j, h in enumerate((2, 2, 8)))     # (the scales would grow)
    ids = i32([1, 0, 2])

    def step():
        c.reserve(ids)                       # sequence 0 needs a new page, and there is none
        for layer in range(2):
            c.append(k, v, ids, layer=layer)
        return c.attention(q, ids, layer=1)

    step()
    raises_at_poll(c, B.ERR_NO_PAGES)
    step()                                    # again, after the poll
    raises_at_poll(c, B.ERR_NO_PAGES)
    c.append(k, v, ids)                       # an append without a new reserve
    raises_at_poll(c, B.ERR_NO_PAGES)
    assert all(torch.equal(a, b) for a, b in zip(before, tensors(c)))
    c.free(i32([3]))
    both.ref.free([3])
    step()
    both.ref.reserve([1, 0, 2], [1, 1, 1])
    for layer in range(2):
        both.ref.append(k.double().cpu().numpy(), v.double().cpu().numpy(), [1, 0, 2], [0, 1, 2, 3], layer)
    both.check_tables()
    both.check_contents()


def test_a_refused_reserve_stops_only_the_sequences_that_it_lists():
    both = Both("e4m3", heads=1, pages=4, max_seqs=4, max_pages=3)
    both.grow([0, 1, 2], [100, 130, 60], 711)
    c = both.gpu
    k = tokens(1, 1, 713).to(DEV)
    before = [t.clone() for t in tensors(c)]
    c.reserve(i32([1, 0, 3]), i32([300, 0, 1]))      # too much for a row; nothing for sequence 0
    c.append(k, k, i32([1]))
    c.append(k, k, i32([1, 1]), i32([0, 1, 1]))
    assert all(torch.equal(a, b) for a, b in zip(before, tensors(c)))
    both.ref.reserve([2], [1])
    c.reserve(i32([2]))
    c.append(k, k, i32([2]))
    both.ref.append(k.double().cpu().numpy(), k.double().cpu().numpy(), [2], [0, 1])
    c.append(k, k, i32([0]))                         # was to grow by nothing: its newest token may be written again
    both.ref.append(k.double().cpu().numpy(), k.double().cpu().numpy(), [0], [0, 1])
    raises_at_poll(c, B.ERR_NO_PAGES)
    c.reserve(i32([1, 1]))                           # listed twice
    c.append(k, k, i32([1]))
    raises_at_poll(c, B.ERR_BAD_CACHE)
    both.check_tables()
    both.check_contents()
    both.grow([1], [3], 715)
    both.check_tables()
    both.check_contents()


def test_a_prompt_that_is_not_the_layer_s_changes_nothing():
    """k or v of another length, number of heads, type or place, or a layer that is not there: the sequence does not grow."""
    from workloads import synth
    both = Both("int8", 1, pages=8, max_seqs=2, max_pages=8, garbage=False)
    both.grow([1], [30], 725)
    q, k, v = synth.random_qkv(300, 4, 1, seed=5, device=DEV)
    layer = crisp.CrispLayer(crisp.make_params(300, 4, 1, sink_tokens=4))
    odd = torch.empty(300 * 128 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(300, 1, 128)
    for bad in ((k[:299], v[:299]), (k, v[:299]), (k, q), (k, v.float()), (k, v.cpu()),
                (k.expand(300, 2, 128).contiguous(), v), (torch.cat([k, k]), torch.cat([v, v]))):
        with pytest.raises(ValueError):
            layer.store(*bad, both.gpu, i32([1]))
    for bad, at in (((k, odd), 0), ((k, v), -1), ((k, v), 1)):
        with pytest.raises(crisp.CrispError):
            layer.store(*bad, both.gpu, i32([1]), cache_layer=at)
    both.check_tables()
    both.check_contents()
    layer.store(k, v, both.gpu, i32([1]))
    both.ref.reserve([1], [300])
    both.ref.append(k.double().cpu().numpy(), v.double().cpu().numpy(), [1], [0, 300])
    both.check_tables()
    both.check_contents()


def test_a_prompt_that_does_not_fit_overwrites_nothing():
    """CrispLayer.store onto a sequence that already holds as many tokens as the prompt has."""
    from workloads import synth
    both = Both("int8", 1, pages=4, max_seqs=2, max_pages=8)
    both.grow([1], [300], 721)
    q, k, v = synth.random_qkv(300, 4, 1, seed=4, device=DEV)
    layer = crisp.CrispLayer(crisp.make_params(300, 4, 1, sink_tokens=4))
    layer.store(k, v, both.gpu, i32([1]))
    raises_at_poll(both.gpu, B.ERR_NO_PAGES)
    both.check_tables()
    both.check_contents()


def test_two_caches_in_one_workspace_do_not_take_each_other_s_refusals():
    """The calls of two caches, one after the other, through one workspace (sized for the larger one)."""
    a = Both("e4m3", heads=1, pages=2, max_seqs=2, max_pages=2)
    b = Both("e4m3", heads=1, pages=90, max_seqs=40, max_pages=4)
    a.gpu._pages_ws, a.gpu.pages_ws = b.gpu._pages_ws, b.gpu.pages_ws
    a.grow([0, 1], [128, 100], 731)
    k = tokens(1, 1, 733).to(DEV)
    a.gpu.reserve(i32([0, 1]))
    a.gpu.append(k, k, i32([0]))
    raises_at_poll(a.gpu, B.ERR_NO_PAGES)
    b.grow(list(range(40)), [1 + 6 * i for i in range(40)], 735)
    b.check_tables()
    b.check_contents()
    a.check_tables()
    a.check_contents()


def test_append_refuses_what_it_must_not_write():
    both = Both("e4m3", heads=1, pages=8, max_seqs=4, max_pages=3)
    both.grow([0], [256], 95)
    both.gpu.fork(i32([0]), i32([1]))
    before = both.gpu.k_codes.clone()
    k = tokens(10, 1, 96).to(DEV)
    for ids, cu in (([0], [0, 10]),        # its last page is shared
                    ([2], [0, 10]),        # more new tokens than it has
                    ([7], [0, 10])):       # no such sequence
        both.gpu.append(k, k, i32(ids), i32(cu))
        with pytest.raises(crisp.CrispError) as e:
            both.gpu.poll()
        assert e.value.status == B.ERR_BAD_CACHE
    both.gpu.append(k, k, i32([0]), i32([0, 11]))   # offsets beyond the tokens
    with pytest.raises(crisp.CrispError):
        both.gpu.poll()
    both.gpu.append(k, k, i32([0]), i32([5, 3]))    # offsets that fall
    with pytest.raises(crisp.CrispError):
        both.gpu.poll()
    assert torch.equal(before, both.gpu.k_codes)


def test_attention_skips_what_breaks_its_rules():
    """Items with a bad description are reported and their rows left alone; the others are computed."""
    both = Both("e4m3", heads=1, pages=8, max_seqs=3, max_pages=3)
    both.grow([0, 1], [200, 90], 97)
    q = tokens(6, 4, 98).to(DEV)
    want = both.gpu.attention(q[:1], i32([0]))
    o = torch.full_like(q, 7.0)
    both.gpu.attention(q, i32([0, 5, 1]), i32([0, 1, 2, 6]), max_new=2, o=o)   # no sequence 5; four tokens are over 2
    with pytest.raises(crisp.CrispError) as e:
        both.gpu.poll()
    assert e.value.status == B.ERR_BAD_CACHE
    assert torch.equal(o[0], want[0]) and (o[1:] == 7).all()
    both.gpu.page_table[0, 1] = 8               # no such page: reported, nothing read beyond the pool
    both.gpu.attention(q[:1], i32([0]))
    with pytest.raises(crisp.CrispError):
        both.gpu.poll()


@pytest.mark.parametrize("length", [-5, 257, 1 << 30])
def test_free_leaves_a_length_that_breaks_its_rule(length):
    both = Both("e4m3", heads=1, pages=4, max_seqs=2, max_pages=2, garbage=False)
    both.grow([0, 1], [128, 5], 745)
    c = both.gpu
    c.seq_lens[0] = length
    before = [t.clone() for t in tensors(c)[:3]]
    c.free(i32([0, 0]))
    raises_at_poll(c, B.ERR_BAD_CACHE)
    assert all(torch.equal(a, b) for a, b in zip(before, tensors(c)[:3]))       # table, lengths, references
    c.seq_lens[0] = 128
    c.free(i32([0, 0]))
    both.ref.free([0])
    both.check_tables()


def test_poll_names_the_errors_of_both_workspaces():
    both = Both("e4m3", heads=1, pages=2, max_seqs=2, max_pages=2)
    both.grow([0, 1], [128, 5], 741)
    c = both.gpu
    c.reserve(i32([0]))                                          # no page
    c.attention(tokens(1, 4, 743).to(DEV), i32([9]))             # no such sequence
    with pytest.raises(crisp.CrispError) as e:
        c.poll()
    assert e.value.status == B.ERR_NO_PAGES
    assert B.status_string(B.ERR_NO_PAGES) in str(e.value) and B.status_string(B.ERR_BAD_CACHE) in str(e.value)
    both.check_tables()


@pytest.mark.parametrize("new,hq", [(1, 8), (4, 64)])
def test_a_call_with_too_much_work_is_refused_as_such(new, hq):
    """Sixteen readers of a sequence of the greatest length, 8 KV heads: 2^31 pages of work.  All of its pages are one page."""
    c = crisp.CrispCache.allocate(1, 8, 1, (1 << 24) - 1)
    c.page_table.zero_()
    c.page_refs.fill_(1)
    c.seq_lens.fill_(((1 << 24) - 1) * 128)
    q = tokens(16 * new, hq, 99).to(DEV)
    o = torch.full_like(q, 7.0)
    c.attention(q, i32([0] * 16), o=o)
    raises_at_poll(c, B.ERR_UNSUPPORTED)
    assert (o == 7).all()


# ------------------------------------------------------------------------------------------------ as they are used
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_prompt_answer_branch_and_compact(fmt):
    """The way of a request: a prompt through Algorithm 1, its K/V into the cache, answer tokens, a branch, the first
    user leaves, the pool is compacted, and the branch answers on.  Attention is checked at every step."""
    from workloads import synth
    w = synth.tiny(n=700)
    q, k, v = synth.make_qkv(w, device=DEV)
    hq, hkv = w.n_q_heads, w.n_kv_heads
    p = crisp.make_params(w.seq_len, hq, hkv, sink_tokens=w.sink_tokens, local_tokens=w.local_tokens)
    layer = crisp.CrispLayer(p)
    layer.forward(q, k, v)
    layer.poll()
    both = Both(fmt, hkv, pages=20, max_seqs=4, max_pages=10)

    def write(ids, cu, k, v):
        n = [b - a for a, b in zip(cu, cu[1:])]
        both.gpu.reserve(i32(ids), i32(n))
        both.gpu.append(k.to(DEV), v.to(DEV), i32(ids), i32(cu))
        both.ref.reserve(ids, n)
        both.ref.append(k.double().cpu().numpy(), v.double().cpu().numpy(), ids, cu)

    layer.store(k, v, both.gpu, i32([0]))
    both.ref.reserve([0], [700])
    both.ref.append(k.double().cpu().numpy(), v.double().cpu().numpy(), [0], [0, 700])
    for step in range(3):
        write([0], [0, 1], tokens(1, hkv, 200 + step), tokens(1, hkv, 210 + step))
        both.check_attention(hq, [0], [1], 220 + step)
    both.gpu.fork(i32([0, 0]), i32([1, 3]), i32([650, 703]))
    both.ref.fork([0, 0], [1, 3], [650, 703])
    write([3, 1, 0], [0, 1, 3, 4], tokens(4, hkv, 230), tokens(4, hkv, 231))
    both.check_attention(hq, [3, 1, 0], [1, 2, 1], 232)
    both.gpu.free(i32([0]))
    both.ref.free([0])
    assert int(both.gpu.compact().item()) == both.ref.compact()
    write([1, 3], [0, 1, 2], tokens(2, hkv, 240), tokens(2, hkv, 241))
    both.check_attention(hq, [1, 3], [1, 1], 242)
    both.check_tables()
    both.check_contents()


def test_a_prompt_of_several_layers_is_stored_once():
    """CrispLayer.store reserves at the first layer and writes each layer's K/V."""
    from workloads import synth
    both = Both("e4m3", 1, pages=8, max_seqs=2, max_pages=4, layers=2)
    q, k, v = synth.random_qkv(300, 4, 1, seed=3, device=DEV)
    layer = crisp.CrispLayer(crisp.make_params(300, 4, 1, sink_tokens=4))
    layer.forward(q, k, v, dense_below_tokens=512)
    for x in range(2):
        layer.store(k * (x + 1), v, both.gpu, i32([1]), cache_layer=x)
    both.ref.reserve([1], [300])
    for x in range(2):
        both.ref.append((k * (x + 1)).double().cpu().numpy(), v.double().cpu().numpy(), [1], [0, 300], layer=x)
    layer.poll()
    both.check_tables()
    both.check_contents()
    # attention of all 300 queries over the stored prompt against the dense kernel on what was given: the codes' rounding
    # (2^-4 of a value for e4m3) is the difference, so only its size is checked
    o = both.gpu.attention(q, i32([1]))
    rel = (o.float() - layer.o.float()).norm() / layer.o.float().norm()
    assert rel < 2.0 ** -4
    with pytest.raises(ValueError):
        layer.store(k, v, both.gpu, i32([0, 1]))


def test_pages_beyond_four_gigabytes():
    """A pool whose code offsets pass 2^32 bytes: the pages in use are its last ones."""
    n_pages = (1 << 32) // (128 * 128) + 40
    both = Both("e4m3", 1, pages=n_pages, max_seqs=3, max_pages=8, garbage=False)
    both.ref.codes = {x: np.zeros((1, 1), np.uint8) for x in "kv"}        # (the reference keeps only the last pages)
    taken = n_pages - 30
    both.gpu.page_refs[:taken] = 1
    small = ref.RefCache(1, 30, 1, 3, 8, "e4m3")
    lens = [700, 130]
    k, v = tokens(830, 1, 401), tokens(830, 1, 402)
    both.gpu.reserve(i32([0, 2]), i32(lens))
    both.gpu.append(k.to(DEV), v.to(DEV), i32([0, 2]), i32([0, 700, 830]))
    both.gpu.fork(i32([0]), i32([1]), i32([650]))
    small.reserve([0, 2], lens)
    small.append(k.double().numpy(), v.double().numpy(), [0, 2], [0, 700, 830])
    small.fork([0], [1], [650])
    both.gpu.poll()
    table = both.gpu.page_table.cpu().numpy()
    assert np.array_equal(np.where(table >= 0, table - taken, -1), small.table)
    for new in (1, 40):
        q = tokens(3 * new, 4, 403 + new)
        lse = torch.empty(4, 3 * new, device=DEV)
        o = both.gpu.attention(q.to(DEV), i32([2, 0, 1]), lse=lse)
        cu = [0, new, 2 * new, 3 * new]
        check_rows(o, lse, small.attention(q.double().numpy(), [2, 0, 1], cu), new * 4)
    both.gpu.poll()


def test_the_largest_batch():
    """1024 sequences of one to three tokens, in one call of each kind."""
    n = B.CACHE_MAX_BATCH
    both = Both("int8", 1, pages=n + 2, max_seqs=n, max_pages=1)
    rng = np.random.RandomState(5)
    lens = rng.randint(1, 4, n).tolist()
    ids = rng.permutation(n).tolist()
    both.grow(ids, lens, 501)
    both.check_tables()
    both.check_attention(2, ids, [1] * n, 502)
    both.check_attention(2, ids, [13 if i % 300 == 0 else 1 for i in range(n)], 503)
    both.gpu.free(i32(ids[::2]))
    both.ref.free(ids[::2])
    assert int(both.gpu.compact().item()) == both.ref.compact()
    both.check_tables()
    both.check_contents()


@pytest.mark.parametrize("seed", range(16))
def test_random_batches(seed):
    """Random shapes, formats, lengths and numbers of new tokens, with padding entries and queries without keys."""
    rng = np.random.RandomState(1000 + seed)
    hkv = int(rng.choice([1, 2, 3]))
    hq = hkv * int(rng.choice([1, 2, 4, 5, 7, 8, 16]))
    batch = int(rng.randint(1, 7))
    top = int(rng.choice([3, 150, 1400]))
    lens = [int(x) for x in rng.randint(0, top + 1, batch)]
    both = Both(str(rng.choice(["e4m3", "int8"])), hkv, pages=batch * 12, max_seqs=batch, max_pages=11)
    both.grow(list(range(batch)), lens, 2000 + 10 * seed, spread=float(rng.choice([0, 6])))
    ids = [int(x) if rng.rand() < 0.85 else -1 for x in rng.permutation(batch)]
    new = [int(x) for x in rng.randint(0, int(rng.choice([1, 3, 20, 260])) + 1, batch)]
    if max(new) == 0:
        new[0] = 1
    both.check_attention(hq, ids, new, 2005 + 10 * seed)


def test_step_in_a_graph_and_on_another_stream():
    """reserve, append and attention of a decode step replay from one CUDA graph as the sequences grow; the same step on
    a side stream gives the same bits."""
    both, other = (Both("e4m3", 2, pages=24, max_seqs=3, max_pages=8) for _ in range(2))
    for b in (both, other):
        b.grow([0, 1, 2], [126, 300, 5], 301)
    ids = i32([2, 0, 1])
    steps = [[tokens(3, h, 310 + 3 * s + j).to(DEV) for j, h in enumerate((8, 2, 2))] for s in range(5)]
    q, k, v = (x.clone() for x in steps[0])
    o = torch.empty_like(q)
    lse = torch.empty(8, 3, device=DEV)

    def step(c):
        c.reserve(ids)
        c.append(k, v, ids)
        c.attention(q, ids, o=o, lse=lse)

    torch.cuda.synchronize()
    state = [t.clone() for t in (both.gpu.page_table, both.gpu.seq_lens, both.gpu.page_refs)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(both.gpu)     # set-up outside the capture
    torch.cuda.synchronize()
    for t, s in zip((both.gpu.page_table, both.gpu.seq_lens, both.gpu.page_refs), state):
        t.copy_(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(both.gpu)
    for s in range(5):
        for dst, src in zip((q, k, v), steps[s]):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = o.clone(), lse.clone()
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        other.gpu.reserve(ids, stream=stream)
        other.gpu.append(steps[s][1], steps[s][2], ids, stream=stream)
        want_lse = torch.empty_like(lse)
        want = other.gpu.attention(steps[s][0], ids, lse=want_lse, stream=stream)
        stream.synchronize()
        assert torch.equal(got, want) and torch.equal(got_lse, want_lse)
    both.gpu.poll()
    other.gpu.poll()
    assert both.gpu.seq_lens.tolist() == [131, 305, 10]


def test_two_graphs_and_two_objects_over_one_cache():
    """Two captured calls that share a workspace, replayed in turn; two objects over the same tensors at the same time."""
    both = Both("int8", 2, pages=120, max_seqs=3, max_pages=60)
    both.grow([0, 1, 2], [7000, 300, 1000], 601)
    c = both.gpu
    twin = crisp.CrispCache(c.k_codes, c.v_codes, c.k_scale, c.v_scale, c.page_table, c.seq_lens, c.page_refs, fmt="int8")
    ids = i32([1, 0, 2])
    jobs = [(tokens(3, 8, 602).to(DEV), 1), (tokens(120, 8, 603).to(DEV), 40), (tokens(9, 8, 604).to(DEV), 3)]
    want = [c.attention(q, ids) for q, _ in jobs]
    out = [torch.empty_like(q) for q, _ in jobs]
    graphs = []
    for (q, _), o in zip(jobs, out):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.attention(q, ids, o=o)
        graphs.append(g)
    for turn in ([0, 1, 2], [2, 2, 1, 0], [1, 0, 1]):
        for o in out:
            o.fill_(7.0)
        for k in turn:
            graphs[k].replay()
        torch.cuda.synchronize()
        for k in set(turn):
            assert torch.equal(out[k], want[k])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[x.attention(q, ids, stream=st) for _ in range(20) for q, _ in jobs] for x, st in zip((c, twin), streams)]
    torch.cuda.synchronize()
    for g in got:
        for i, o in enumerate(g):
            assert torch.equal(o, want[i % 3])
    c.poll()
    twin.poll()


def test_outputs_belong_to_the_stream_that_writes_them():
    """An output that the call allocates for a stream given as a handle is not memory that the current stream still reads."""
    both = Both("e4m3", 2, pages=4, max_seqs=1, max_pages=4)
    both.grow([0], [300], 611)
    c, ids, q = both.gpu, i32([0]), tokens(300, 8, 612).to(DEV)
    want = c.attention(q, ids)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for call, like in ((lambda: c.attention(q, ids, stream=side.cuda_stream), q),
                       (lambda: c.compact(stream=side.cuda_stream), torch.empty(1, dtype=torch.int32, device=DEV))):
        old = torch.full_like(like, 7)
        seen = torch.empty_like(like)
        torch.cuda.synchronize()
        torch.cuda._sleep(100_000_000)     # keeps the current stream busy for some tens of milliseconds
        seen.copy_(old)
        del old
        out = call()
        torch.cuda.synchronize()
        assert (seen == 7).all()
        assert torch.equal(out, want) if out.shape == want.shape else out.item() == 3
    c.poll()


@pytest.mark.parametrize("handle", [False, True])
def test_inputs_may_be_dropped_behind_a_call_on_another_stream(handle):
    """The side stream is busy when the calls are made; their temporaries' memory is not handed out again before they ran."""
    both = Both("e4m3", 2, pages=8, max_seqs=2, max_pages=4)
    both.grow([1], [10], 621)
    c = both.gpu
    k, v, q = (tokens(300, h, 623 + j) for j, h in enumerate((2, 2, 8)))
    both.ref.reserve([0], [300])
    both.ref.append(k.double().numpy(), v.double().numpy(), [0], [0, 300])
    side = torch.cuda.Stream()
    stream = side.cuda_stream if handle else side
    given = [x.to(DEV) for x in (k, v, q)]
    lse = torch.full((8, 300), 7.0, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)     # some tens of milliseconds
    ids, n_new, cu, temporary = i32([0]), i32([300]), i32([0, 300]), [x.clone() for x in given]
    side.wait_stream(torch.cuda.current_stream())
    c.reserve(ids, n_new, stream=stream)
    c.append(*temporary[:2], ids, cu, stream=stream)
    o = c.attention(temporary[2], ids, lse=lse, stream=stream)
    del ids, n_new, cu, temporary
    junk = [torch.full_like(x, float("nan")) for x in given for _ in range(3)] + [i32([1]) for _ in range(20)]
    junk += [i32([0, 5]) for _ in range(20)]
    torch.cuda.synchronize()
    both.check_tables()
    both.check_contents()
    check_rows(o, lse, both.ref.attention(q.double().numpy(), [0], [0, 300]), 1200)
    del junk


def test_handle_zero_is_the_default_stream():
    """Outputs that a call allocates for stream=0, with another stream current, come from the default stream's memory."""
    both = Both("e4m3", 2, pages=40, max_seqs=1, max_pages=40)
    both.grow([0], [5000], 613)
    ids, q = i32([0]), tokens(5000, 8, 614).to(DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        outs = [both.gpu.attention(q, ids, stream=0), both.gpu.compact(stream=0)]
    torch.cuda.synchronize()
    for out in outs:
        at = out.data_ptr()
        home = [x["stream"] for x in torch.cuda.memory_snapshot() if x["address"] <= at < x["address"] + x["total_size"]]
        assert home == [torch.cuda.default_stream().cuda_stream] == [0]
    both.gpu.poll(stream=0)


def test_the_binding_s_calls_are_the_object_s():
    """The functions of binding.py on a descriptor do what the methods do."""
    a, b = (Both("int8", 2, pages=16, max_seqs=4, max_pages=4, garbage=False) for _ in range(2))
    ids, n_new, cu = i32([1, 3]), i32([200, 5]), i32([0, 200, 205])
    q, k, v = (tokens(205, h, 620 + h + j).to(DEV) for j, h in enumerate((8, 2, 2)))
    src, dst, cut = i32([1]), i32([0]), i32([150])
    c, d = a.gpu, b.gpu
    c.reserve(ids, n_new)
    c.append(k, v, ids, cu)
    want = c.attention(q, ids, cu)
    c.fork(src, dst, cut, share=False)
    c.free(ids[1:])
    used = c.compact()
    o, lse, n = torch.empty_like(q), torch.empty(8, 205, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    assert B.crisp_cache_reserve(d.desc, ids, n_new, 2, d.pages_ws) == B.OK
    assert B.crisp_cache_append(d.desc, 0, ids, cu, 2, 205, k, v, d.pages_ws) == B.OK
    assert B.crisp_cache_attention(d.desc, 0, ids, cu, 2, 205, 205, 8, 0.0, q, o, lse, d.attention_ws) == B.OK
    assert B.crisp_cache_fork(d.desc, src, dst, cut, 1, False, d.pages_ws) == B.OK
    assert B.crisp_cache_free(d.desc, ids[1:], 1, d.pages_ws) == B.OK
    assert B.crisp_cache_compact(d.desc, n, d.pages_ws) == B.OK
    c.poll()
    d.poll()
    assert torch.equal(o, want) and n.item() == used.item() == 4
    for name in ("page_table", "seq_lens", "page_refs"):
        assert torch.equal(getattr(c, name), getattr(d, name))


def test_arguments_are_checked():
    c = crisp.CrispCache.allocate(4, 2, 2, 2)
    q = tokens(2, 4, 1).to(DEV)
    ids = i32([0, 1])
    for bad in (lambda: c.attention(q.float(), ids), lambda: c.attention(q.transpose(0, 1), ids),
                lambda: c.attention(q, ids.long()), lambda: c.attention(q, ids, i32([0, 2])),
                lambda: c.attention(q.cpu(), ids), lambda: c.attention(q, ids, lse=torch.empty(2, 4, device=DEV)),
                lambda: c.attention(q, ids, o=q[:1]), lambda: c.append(q, q, ids), lambda: c.reserve(ids, i32([1])),
                lambda: c.append(q[:, :2].contiguous(), q[:1, :2].contiguous(), ids),
                lambda: c.fork(ids, i32([0])), lambda: c.free(ids[::2].expand(2)),
                lambda: crisp.CrispCache(c.k_codes, c.v_codes, c.k_scale, c.v_scale, c.page_table, c.seq_lens,
                                         c.page_refs, fmt="fp4"),
                lambda: crisp.CrispCache(c.k_codes, c.v_codes[:, :3], c.k_scale, c.v_scale, c.page_table, c.seq_lens,
                                         c.page_refs)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: c.attention(q, ids, layer=1), lambda: c.attention(q, ids, softmax_scale=-1.0),
                lambda: c.attention(q, ids, max_new=0), lambda: c.attention(tokens(3, 4, 1).to(DEV), ids),
                lambda: c.attention(tokens(2, 3, 1).to(DEV), ids), lambda: c.attention(tokens(2, 34, 1).to(DEV), ids)):
        with pytest.raises(crisp.CrispError):
            bad()
    c.attention(q[:0], ids[:0])            # nothing to do
    c.reserve(ids[:0])
    c.free(ids[:0])
    c.poll()
