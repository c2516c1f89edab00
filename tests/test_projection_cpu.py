"""The operators around the attention, without a GPU: refusals, the plan's layout and frequencies, and the reference that the
GPU tests compare with, checked against closed forms."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2609_01925_b200 as crisp
from paper_2609_01925_b200 import binding as B
from tests import projection_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, ODD, WORD = 0x1000, 0x100a, 0x1004      # never dereferenced: validation comes first
NAN, INF = float("nan"), float("inf")


def test_quantize_refusals():
    lib = B.load()

    def call(x=FAKE, rows=4, cols=256, codes=FAKE, scales=FAKE):
        return lib.crisp_quantize(x, rows, cols, codes, scales, None)

    assert call(x=None) == call(codes=None) == call(scales=None) == B.ERR_INVALID_ARG
    assert call(x=ODD) == call(codes=ODD) == call(scales=ODD) == call(rows=-1) == call(cols=0) == call(cols=-16) == B.ERR_INVALID_ARG
    assert call(cols=250) == call(cols=(1 << 28) + 16) == call(rows=(1 << 28) + 1) == B.ERR_UNSUPPORTED
    assert call(rows=0) == call(rows=0, x=None) == B.OK


def test_norm_refusals():
    lib = B.load()

    def call(x=FAKE, residual=None, weight=FAKE, rows=4, cols=256, eps=1e-5, total=None, y=FAKE, codes=None, scales=None):
        return lib.crisp_rms_norm(x, residual, weight, rows, cols, eps, total, y, codes, scales, None)

    bad = [dict(x=None), dict(x=ODD), dict(weight=ODD), dict(y=ODD), dict(y=None), dict(codes=FAKE, scales=FAKE), dict(y=None, codes=FAKE),
           dict(scales=FAKE), dict(residual=FAKE), dict(total=FAKE), dict(residual=ODD, total=FAKE), dict(residual=FAKE, total=ODD),
           dict(eps=-1e-9), dict(eps=NAN), dict(eps=INF), dict(rows=-1), dict(cols=0), dict(y=None, codes=ODD, scales=FAKE)]
    for kw in bad:
        assert call(**kw) == B.ERR_INVALID_ARG, kw
    assert call(cols=24) == call(cols=32784) == B.ERR_UNSUPPORTED
    assert call(rows=0) == B.OK


def test_matmul_refusals():
    lib = B.load()
    size = B.crisp_matmul_workspace_bytes()
    assert size >= 256

    def call(codes=FAKE, scales=FAKE, w=FAKE, ws_=FAKE, rows=4, n=128, cols=256, out=FAKE, ws=FAKE, ws_bytes=size):
        return lib.crisp_matmul(codes, scales, w, ws_, rows, n, cols, out, ws, ws_bytes, None)

    for kw in (dict(codes=None), dict(scales=None), dict(w=None), dict(ws_=None), dict(out=None), dict(ws=None), dict(codes=ODD),
               dict(codes=WORD), dict(w=WORD), dict(out=WORD),
               dict(scales=ODD), dict(w=ODD), dict(ws_=ODD), dict(out=ODD), dict(rows=-1), dict(n=-1), dict(cols=0)):
        assert call(**kw) == B.ERR_INVALID_ARG, kw
    assert call(cols=8) == call(cols=1 << 29) == call(rows=1 << 29) == call(n=1 << 29) == B.ERR_UNSUPPORTED
    assert call(ws=ODD) == call(ws_bytes=size - 1) == B.ERR_WORKSPACE
    assert call(rows=0) == call(n=0) == B.OK


def test_rotary_plan_matches_the_header():
    header = open(os.path.join(ROOT, "include", "crisp.h")).read()
    body = header[header.index("typedef struct crisp_rotary_plan {"):header.index("} crisp_rotary_plan;")]
    fields = re.findall(r"^\s*(?:int32_t|float|uint64_t)\s+(\w+)(?:\[64\])?;", body, flags=re.M)
    assert fields == [f[0] for f in B.CrispRotaryPlan._fields_]
    assert ctypes.sizeof(B.CrispRotaryPlan) == 4 * 4 + 64 * 8
    for name, value in re.findall(r"#define CRISP_(ROTARY_\w+) (\d+)", header):
        assert getattr(B, name) == int(value)


@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                dict(scaling="ramp", factor=8.0, original=8192), dict(scaling="bands", factor=8.0, original=8192),
                                dict(scaling="ramp", factor=2.0, original=300, low=2.0, high=9.0),
                                dict(scaling="bands", factor=16.0, original=100, low=0.5, high=3.0)])
@pytest.mark.parametrize("dim,theta", [(16, 10000.0), (96, 1e6), (128, 500000.0)])
def test_rotary_frequencies(kw, dim, theta):
    plan = crisp.CrispRotary(theta, rotary_dim=dim, **kw).plan
    want = ref.frequencies(dim, theta, **kw)
    for i, f in enumerate(want):
        # a whole number of 2^-64 turns: half of one off, besides the roundings of a few float64 operations
        assert abs(plan.turns[i] / 2.0 ** 64 * 2 * math.pi - f) <= 2.0 ** -49 * f + math.pi * 2.0 ** -64
    assert all(t == 0 for t in plan.turns[dim // 2:])
    assert plan.magnitude == np.float32(0.1 * math.log(kw["factor"]) + 1.0 if kw.get("scaling") == "ramp" else 1.0)


def test_rotary_refusals():
    for kw in (dict(theta=1.0), dict(theta=NAN), dict(theta=INF), dict(rotary_dim=0), dict(rotary_dim=24), dict(rotary_dim=144),
               dict(scaling="linear", factor=0.5), dict(factor=NAN), dict(scaling="ramp", factor=2.0),
               dict(scaling="bands", factor=2.0, original=-5), dict(scaling="bands", factor=2.0, original=100, low=4.0, high=4.0)):
        with pytest.raises(crisp.CrispError):
            crisp.CrispRotary(**{"theta": 1e4, **kw})
    for kw in (dict(layout="other"), dict(scaling="other")):
        with pytest.raises(ValueError):
            crisp.CrispRotary(1e4, **kw)
    lib = B.load()
    plan = B.crisp_rotary_init(128, B.ROTARY_HALF, 1e4)

    def call(plan=plan, n=4, hq=4, hkv=1, q=FAKE, qs=768, k=FAKE, ks=768, v=FAKE, vs=768, qo=FAKE + 64, ko=FAKE + 64, vo=FAKE + 64):
        return lib.crisp_rotary(ctypes.byref(plan), n, None, 0, hq, hkv, q, qs, k, ks, v, vs, qo, ko, vo, None)

    for kw in (dict(n=-1), dict(hq=-1), dict(q=None), dict(qo=None), dict(k=ODD), dict(vo=ODD), dict(qs=504), dict(qs=516), dict(ks=64),
               dict(hq=0), dict(hkv=0), dict(qo=FAKE), dict(vs=1 << 40)):
        assert call(**kw) == B.ERR_INVALID_ARG, kw
    assert call(n=(1 << 28) + 1) == call(hq=65536, qs=1 << 24) == B.ERR_UNSUPPORTED
    assert call(n=0) == call(q=None, qo=None, k=None, ko=None, v=None, vo=None) == B.OK
    for name, value, code in (("struct_size", 8, B.ERR_INVALID_ARG), ("layout", 2, B.ERR_INVALID_ARG), ("rotary_dim", 8, B.ERR_UNSUPPORTED),
                              ("rotary_dim", 0, B.ERR_INVALID_ARG), ("magnitude", NAN, B.ERR_INVALID_ARG)):
        other = B.CrispRotaryPlan.from_buffer_copy(plan)
        setattr(other, name, value)
        assert call(plan=other) == code


def test_no_cpu_fallback():
    x = torch.zeros(2, 256, dtype=torch.bfloat16)
    for bad in (lambda: crisp.quantize(x), lambda: crisp.rms_norm(x), lambda: crisp.CrispRotary(1e4).split(x, 1, 1),
                lambda: crisp.CrispRotary(1e4).rotate(x.view(2, 2, 128)),
                lambda: crisp.CrispLinear(x.to(torch.float8_e4m3fn), torch.zeros(2, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu))):
        with pytest.raises(RuntimeError):
            bad()


# ------------------------------------------------------------------------------------------------ the reference itself
def test_reference_operands():
    assert ref.exponent(448.0) == 0 and ref.exponent(449.0) == 1 and ref.exponent(224.0) == -1 and ref.exponent(0.0) == -126
    assert ref.exponent(2.0 ** -130) == -126
    v = np.concatenate([np.linspace(-448, 448, 4001), [17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 0.0]])
    want = torch.tensor(v).to(torch.float8_e4m3fn)
    np.testing.assert_array_equal(np.array(ref.E4M3)[ref.encode(v)], want.double().numpy())
    assert (np.abs(want.double().numpy() - v) <= ref.half_step(v)).all()
    x = np.random.RandomState(0).randn(3, 700)
    codes, scales = ref.quantize(x)
    assert scales.shape == (3, 8) and (scales[:, 6:] == 127).all()
    assert (np.abs(ref.values(codes, scales) - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -16)).all()


def test_reference_rounds_once():
    x = np.array([1 + 2.0 ** -8, 1 + 2.0 ** -8 + 2.0 ** -40, 1 + 3 * 2.0 ** -8 - 2.0 ** -40, -(1 + 2.0 ** -8 + 2.0 ** -40), 0.1])
    np.testing.assert_array_equal(ref.bf16(x)[:4], [1.0, 1 + 2.0 ** -7, 1 + 2.0 ** -7, -(1 + 2.0 ** -7)])


def test_reference_norm_and_rotary():
    x = np.random.RandomState(1).randn(2, 64)
    y, h = ref.norm(x, None, None, 0.0)
    np.testing.assert_allclose((y * y).mean(1), 1.0)
    assert h is x
    x = np.random.RandomState(2).randn(3, 1, 128)
    freq = ref.frequencies(128, 1e4)
    assert freq[0] == 1.0 and abs(freq[-1] - 1e4 ** (-126 / 128)) < 1e-15
    r = ref.rotate(x, [0, 3, 7], freq, "half")
    np.testing.assert_array_equal(r[0], x[0])
    np.testing.assert_allclose(r[1, 0, 0], x[1, 0, 0] * math.cos(3) - x[1, 0, 64] * math.sin(3))
    np.testing.assert_allclose(r[1, 0, 64], x[1, 0, 64] * math.cos(3) + x[1, 0, 0] * math.sin(3))
    # scores depend on distances alone
    a, b = (ref.rotate(x, [p, p + 4, p + 9], freq, "interleaved")[:, 0] for p in (0, 100))
    np.testing.assert_allclose(a @ a.T, b @ b.T)


# ------------------------------------------------------------------------------------------------ the product's ring of stages
def run_ring(stages, loaders, issuers, steps, seed):
    """The loading and issuing warps of the product over one ring, in a random order: barriers know the parity of their phase
    only, copies land late, products free their stage late (in order, for one issuer).  Returns what went wrong, or None."""
    rng = np.random.RandomState(seed)
    full, empty = [0] * stages, [0] * stages            # phases that have ended
    holds, freed = [None] * stages, [0] * stages        # step in the stage, uses that have ended
    load_at, issue_at = list(range(loaders)), list(range(issuers))
    landing, running = [], [[] for _ in range(issuers)]
    passed = lambda ended, parity: (ended & 1) != parity  # noqa: E731
    for _ in range(60 * steps):
        kind = rng.randint(4)
        if kind == 0:
            w = rng.randint(loaders)
            i = load_at[w]
            st, use = i % stages, i // stages
            if i < steps and (i < stages or passed(empty[st], (use - 1) & 1)):
                if freed[st] != use:
                    return f"step {i} is loaded over a stage in use"
                landing.append(i)
                load_at[w] += loaders
        elif kind == 1 and landing:
            i = landing.pop(rng.randint(len(landing)))
            holds[i % stages] = i
            full[i % stages] += 1
        elif kind == 2:
            w = rng.randint(issuers)
            i = issue_at[w]
            if i < steps and passed(full[i % stages], (i // stages) & 1):
                if holds[i % stages] != i:
                    return f"step {i} finds step {holds[i % stages]}"
                running[w].append(i)
                issue_at[w] += issuers
        elif kind == 3:
            w = rng.randint(issuers)
            if running[w]:
                i = running[w].pop(0)
                empty[i % stages] += 1
                freed[i % stages] += 1
        if min(load_at) >= steps and min(issue_at) >= steps and not any(running):
            return None
    return None if sum(freed) == steps else "no end"


@pytest.mark.parametrize("stages", [2, 3, 4, 5, 6, 8, 11, 12])
def test_ring_of_the_product(stages):
    """Two loading warps that take turns and one that issues, as in matmul.cu and matmul_pair.cu."""
    for seed in range(150):
        assert run_ring(stages, 2, 1, 5 * stages + 3, seed) is None


@pytest.mark.parametrize("stages,loaders,issuers", [(3, 4, 1), (4, 3, 2), (5, 4, 2)])
def test_the_ring_model_sees_loaders_that_come_too_early(stages, loaders, issuers):
    assert any(run_ring(stages, loaders, issuers, 5 * stages + 3, seed) for seed in range(400))


@pytest.mark.parametrize("way", ["copy", "deepcopy", "pickle"])
def test_a_copied_rotary_uses_its_own_plan(way, monkeypatch):
    """The address that a call is given is that of the plan the object holds, whatever became of the object it was made from."""
    import copy
    import ctypes
    import pickle
    given = []

    class Calls:
        def rotary_split(self, plan, *rest):
            given.append(plan)

        def rotary_rotate(self, plan, *rest):
            given.append(plan)

    monkeypatch.setattr(crisp.binding, "calls", Calls)
    first = crisp.CrispRotary(1e4, rotary_dim=64)
    made = {"copy": copy.copy, "deepcopy": copy.deepcopy, "pickle": lambda r: pickle.loads(pickle.dumps(r))}[way](first)
    assert bytes(made.plan) == bytes(first.plan)
    made.split(None, 4, 1)
    made.rotate(None)
    made.plan = crisp.CrispRotary(5e5).plan
    made.split(None, 4, 1)
    assert given[2] == ctypes.addressof(made.plan) and given[0] == given[1]
    if way != "copy":
        assert given[0] != ctypes.addressof(first.plan)


@pytest.mark.parametrize("kw", [dict(low=0.0), dict(high=0.0), dict(low=0), dict(low=float("nan"))])
@pytest.mark.parametrize("scaling", ["ramp", "bands"])
def test_turns_of_zero_are_refused(scaling, kw):
    """None stands for the usual turns; zero is not taken for it."""
    with pytest.raises((ValueError, RuntimeError)):
        crisp.CrispRotary(5e5, scaling=scaling, factor=8.0, original=8192, **kw)


def test_a_tile_of_many_columns_is_waited_for(tmp_path):
    """The warps that write a tile wait for all of its columns: ten times as long as the product's own estimates say that a tile of
    any documented size takes (pairs: 95 + 0.9 ns per token for a block, 224 tokens; a CTA alone: 520 ns), five times where CTAs
    crowd an SM (four times as long)."""
    import subprocess
    source = tmp_path / "wait.cpp"
    source.write_text('#include <cstdio>\n#include <cstdlib>\n#include "matmul_wait.h"\n'
                      'int main(int n, char** a) { for (int i = 1; i < n; ++i) std::printf("%llu ", crisp::tile_wait_ns(std::atoi(a[i]))); }\n')
    exe = str(tmp_path / "wait")
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2609_01925_b200", "csrc"), "-o", exe, str(source)], check=True)
    blocks = [1, 64, 16383, 16384, 100000, 1 << 20, 1 << 21]
    waits = [int(w) for w in subprocess.run([exe, *map(str, blocks)], check=True, capture_output=True, text=True).stdout.split()]
    for b, w in zip(blocks, waits):
        assert w >= 10 * b * (95 + 0.9 * 224) and w >= 10 * b * 520 and w >= 5 * b * 520 * 4
    assert waits[:3] == [400_000_000] * 3


def test_norm_refuses_one_place_for_two_outputs():
    """The sum and the result over the same memory would leave one of them."""
    lib = B.load()
    for y, codes, scales in ((FAKE, None, None), (None, FAKE, 2 * FAKE)):
        assert lib.crisp_rms_norm(3 * FAKE, 4 * FAKE, None, 4, 256, 1e-5, FAKE, y, codes, scales, None) == B.ERR_INVALID_ARG
        assert lib.crisp_rms_norm(FAKE, 4 * FAKE, None, 4, 256, 1e-5, FAKE, y, codes, scales, None) == B.ERR_INVALID_ARG


def test_the_compiled_calls_belong_to_their_torch(monkeypatch):
    """Beside another torch or Python the module that was built for this one is neither loaded nor taken for up to date."""
    import sys
    import types
    from paper_2609_01925_b200 import build
    here = build.calls_path()
    assert os.path.exists(here) and B.calls()
    monkeypatch.setattr(B, "_calls", None)
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "0.0.1+other")
        assert build.calls_path() != here and build.needs_build()
        with pytest.raises(ImportError):
            B.calls()
    with monkeypatch.context() as m:
        m.setattr(sys, "implementation", types.SimpleNamespace(**{**vars(sys.implementation), "cache_tag": "other-99"}))
        assert build.calls_path() != here and build.needs_build()
        with pytest.raises(ImportError):
            B.calls()
    assert build.calls_path() == here and B.calls()
