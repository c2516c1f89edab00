"""The paged 8-bit cache, without a GPU: host-side refusals, the descriptor's layout, and the reference cache that the
GPU tests compare with, checked against closed forms."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_01925_b200 as crisp
from paper_2609_01925_b200 import binding as B
from tests import cache_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, ODD = 0x1000, 0x1004      # never dereferenced: validation comes first


def desc(**kw):
    base = dict(struct_size=ctypes.sizeof(B.CrispCacheDesc), format=0, n_layers=2, n_kv_heads=8, n_pages=100, max_seqs=4,
                max_pages=10, head_dim=128, k_codes=FAKE, v_codes=FAKE, k_scale=FAKE, v_scale=FAKE, page_table=FAKE,
                seq_lens=FAKE, page_refs=FAKE)
    base.update(kw)
    return B.CrispCacheDesc(**base)


def test_descriptor_matches_the_header():
    header = open(os.path.join(ROOT, "include", "crisp.h")).read()
    body = header[header.index("typedef struct crisp_cache {"):header.index("} crisp_cache;")]
    fields = re.findall(r"^\s*(?:int32_t\*?|float\*?|void\*)\s+(\w+);", body, flags=re.M)
    assert fields == [f[0] for f in B.CrispCacheDesc._fields_]
    assert ctypes.sizeof(B.CrispCacheDesc) == 8 * 4 + 7 * 8
    assert int(re.search(r"#define CRISP_CACHE_MAX_BATCH (\d+)", header).group(1)) == B.CACHE_MAX_BATCH


@pytest.mark.parametrize("kw,code", [
    (dict(struct_size=8), B.ERR_INVALID_ARG), (dict(format=2), B.ERR_INVALID_ARG), (dict(n_layers=0), B.ERR_INVALID_ARG),
    (dict(n_pages=-1), B.ERR_INVALID_ARG), (dict(head_dim=64), B.ERR_UNSUPPORTED), (dict(max_seqs=0), B.ERR_INVALID_ARG),
    (dict(max_pages=1 << 24), B.ERR_UNSUPPORTED), (dict(n_pages=1 << 20), B.ERR_UNSUPPORTED),
    (dict(k_codes=ODD), B.ERR_INVALID_ARG), (dict(v_codes=None), B.ERR_INVALID_ARG), (dict(page_refs=None), B.ERR_INVALID_ARG),
])
def test_bad_descriptors_are_refused(kw, code):
    with pytest.raises(crisp.CrispError) as e:
        B.crisp_cache_workspace_bytes(desc(**kw))
    assert e.value.status == code
    lib = B.load()
    d = ctypes.byref(desc(**kw))
    assert lib.crisp_cache_reserve(d, FAKE, None, 1, FAKE, 1 << 30, None) == code
    assert lib.crisp_cache_append(d, 0, FAKE, None, 1, 1, FAKE, FAKE, FAKE, 1 << 30, None) == code
    assert lib.crisp_cache_attention(d, 0, FAKE, None, 1, 1, 1, 8, 0.0, FAKE, FAKE, None, FAKE, 1 << 30, None) == code
    assert lib.crisp_cache_fork(d, FAKE, FAKE, None, 1, 1, FAKE, 1 << 30, None) == code
    assert lib.crisp_cache_free(d, FAKE, 1, FAKE, 1 << 30, None) == code
    assert lib.crisp_cache_compact(d, FAKE, FAKE, 1 << 30, None) == code


def test_bad_arguments_are_refused():
    lib = B.load()
    d = ctypes.byref(desc())
    pages_ws, attention_ws = B.crisp_cache_workspace_bytes(desc())
    assert pages_ws > 256 and attention_ws > 256
    big = 1 << 40

    def attention(layer=0, cu=None, batch=2, n=2, max_new=1, hq=8, scale=0.0, q=FAKE, o=FAKE, ws=FAKE, ws_bytes=big):
        return lib.crisp_cache_attention(d, layer, FAKE, cu, batch, n, max_new, hq, scale, q, o, None, ws, ws_bytes, None)

    assert attention(layer=2) == attention(layer=-1) == B.ERR_INVALID_ARG
    assert attention(n=3) == attention(n=-2) == attention(max_new=0) == attention(max_new=-1) == B.ERR_INVALID_ARG
    assert attention(batch=-1) == B.ERR_INVALID_ARG
    assert attention(batch=1025, n=1025) == B.ERR_UNSUPPORTED
    assert attention(hq=9) == attention(hq=0) == B.ERR_INVALID_ARG
    assert attention(hq=8 * 17) == B.ERR_UNSUPPORTED
    assert attention(scale=-1.0) == attention(scale=float("nan")) == attention(scale=float("inf")) == B.ERR_INVALID_ARG
    assert attention(q=None) == attention(o=ODD) == attention(ws=None) == B.ERR_INVALID_ARG
    assert attention(ws=ODD) == attention(ws_bytes=attention_ws - 1) == B.ERR_WORKSPACE
    assert attention(batch=0, n=0) == B.OK          # nothing to do, nothing launched

    def append(layer=0, batch=2, n=2, k=FAKE, v=FAKE, ws=FAKE, ws_bytes=big):
        return lib.crisp_cache_append(d, layer, FAKE, None, batch, n, k, v, ws, ws_bytes, None)

    assert append(layer=2) == append(n=3) == append(k=None) == append(v=ODD) == append(ws=None) == B.ERR_INVALID_ARG
    assert append(ws_bytes=pages_ws - 1) == B.ERR_WORKSPACE
    assert append(batch=0, n=0) == append(n=0) == B.OK
    assert lib.crisp_cache_reserve(d, FAKE, None, -1, FAKE, big, None) == B.ERR_INVALID_ARG
    assert lib.crisp_cache_reserve(d, FAKE, None, 1025, FAKE, big, None) == B.ERR_UNSUPPORTED
    assert lib.crisp_cache_reserve(d, FAKE, None, 1, ODD, big, None) == B.ERR_WORKSPACE
    assert lib.crisp_cache_reserve(d, FAKE, None, 0, FAKE, big, None) == B.OK
    assert lib.crisp_cache_fork(d, None, FAKE, None, 1, 1, FAKE, big, None) == B.ERR_INVALID_ARG
    assert lib.crisp_cache_free(d, None, 1, FAKE, big, None) == B.ERR_INVALID_ARG
    assert lib.crisp_cache_compact(d, None, FAKE, big, None) == B.ERR_INVALID_ARG


def test_cache_refuses_to_run_without_cuda():
    if torch.cuda.is_available():
        pytest.skip("CUDA present")
    with pytest.raises(RuntimeError):
        crisp.CrispCache.allocate(4, 1, 1, 4)
    codes, scale = torch.zeros(1, 4, 1, 128, 128, dtype=torch.uint8), torch.zeros(1, 4, 1)
    with pytest.raises(RuntimeError):
        crisp.CrispCache(codes, codes, scale, scale, torch.zeros(1, 4, dtype=torch.int32),
                         torch.zeros(1, dtype=torch.int32), torch.zeros(4, dtype=torch.int32))


# ------------------------------------------------------------------------------------------------ the tile kernel's rings
def ring_model(tmp_path, *flags):
    """Output of cache_ring_model.cpp, built with the kernel's own constants."""
    exe = str(tmp_path / "model")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2609_01925_b200", "csrc"), *flags, "-o", exe,
                    os.path.join(ROOT, "tests", "cache_ring_model.cpp")], check=True)
    return subprocess.run([exe], check=True, capture_output=True, text=True, timeout=120).stdout.strip()


def test_converters_never_take_another_load_s_codes(tmp_path):
    """Copies that land late or out of order do not let a pair of converter warps pass a barrier's earlier phase."""
    assert ring_model(tmp_path) == "ok"


def test_the_ring_model_sees_a_slot_that_changes_hands(tmp_path):
    """Loads dealt in turns of two: a slot of six changes hands, and its new pair takes the parity of a phase that it has not
    seen for the one it waits for."""
    assert "(seed" in ring_model(tmp_path, "-DOWNER(load)=((load)>>1&1u)")


# ------------------------------------------------------------------------------------------------ the reference itself
def test_reference_formats():
    assert ref.E4M3[0x7e] == 448 and ref.E4M3[1] == 2.0 ** -9 and ref.E4M3[0xb8] == -1.0 and np.isnan(ref.E4M3[0x7f])
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ref.E4M3, t)
    x = np.concatenate([np.linspace(-448, 448, 20011), [17.0, 18.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -10, 0.0]])
    want = torch.tensor(x).to(torch.float8_e4m3fn).double().numpy()      # nearest, ties to even
    np.testing.assert_array_equal(ref.values(ref.encode(x, "e4m3"), "e4m3"), want)
    np.testing.assert_array_equal(ref.values(ref.encode([0.5, 1.5, -2.5, 300, np.nan], "int8"), "int8"), [0, 2, -2, 127, 0])
    for fmt, top in ref.LARGEST.items():
        for e in (-126, -3, 0, 90):
            assert ref.exponent(top * 2.0 ** e, fmt) == e and ref.exponent(top * 2.0 ** e * (1 + 2.0 ** -7), fmt) == e + 1
        assert ref.exponent(0.0, fmt) == -126


def test_reference_attention_closed_forms():
    """Equal keys: the mean of the visible values; one key far ahead: its value; nothing visible: zeros."""
    v = np.random.RandomState(0).randn(5, 1, 128)
    k = np.zeros((5, 1, 128))
    q = np.ones((2, 2, 128))
    o, lse, _, _ = ref.attention(lambda s: (k, v), q, [0], [0, 2])
    np.testing.assert_allclose(o[0, 1], v[:4, 0].mean(0))
    np.testing.assert_allclose(o[1, 0], v[:, 0].mean(0))
    np.testing.assert_allclose(lse, np.log([[4, 5], [4, 5]]))
    k[2] = 100.0
    o, _, _, _ = ref.attention(lambda s: (k, v), q, [0], [0, 2])
    np.testing.assert_allclose(o[1, 0], v[2, 0])
    o, lse, _, _ = ref.attention(lambda s: (k[:1], v[:1]), q, [0], [0, 2])
    assert (o[0] == 0).all() and (lse[:, 0] == -np.inf).all() and (o[1] == v[0]).all()


def test_reference_pages():
    c = ref.RefCache(1, 6, 1, 4, 4, "int8")
    c.reserve([1, 0], [130, 1])
    assert c.table[1, :2].tolist() == [0, 1] and c.table[0, 0] == 2 and c.refs.tolist() == [1, 1, 1, 0, 0, 0]
    c.fork([1], [3])
    assert c.table[3, :2].tolist() == [0, 3] and c.refs.tolist() == [2, 1, 1, 1, 0, 0]
    with pytest.raises(ref.Refused):
        c.reserve([2], [257])
    c.free([1, 1])
    assert c.refs.tolist() == [1, 0, 1, 1, 0, 0] and c.lens.tolist() == [1, 0, 0, 130]
    assert c.compact() == 3 and c.table[3, :2].tolist() == [0, 1] and c.refs.tolist() == [1, 1, 1, 0, 0, 0]
