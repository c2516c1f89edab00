"""The operators around the attention on the GPU against float64 (projection_reference.py): quantising is exact; the norm,
the product and the rotary positions stay within bounds derived from their roundings."""
import numpy as np
import pytest
import torch

import paper_2609_01925_b200 as crisp
from tests import projection_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
HALF_BF16 = 2.0 ** -8     # half a step of bf16, relative


def normal(*shape, seed=0, spread=0.0):
    """bf16 on the CPU; with `spread` rows of blocks differ by powers of two up to 2^spread."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g)
    if spread:
        x = x * torch.exp2(torch.rand(*shape[:-1], 1, generator=g) * spread - spread / 2)
    return x.bfloat16()


def f64(t):
    return t.detach().cpu().double().numpy()


def raw(t):
    return t.view(torch.uint8).cpu().numpy()


# ------------------------------------------------------------------------------------------------ 8-bit operands
@pytest.mark.parametrize("rows,cols", [(1, 16), (1, 128), (3, 144), (5, 512), (2, 528), (7, 2048), (9, 2064), (1, 4096),
                                       (37, 3584), (300, 48), (2, 20000)])
def test_quantize_is_exact(rows, cols):
    x = normal(rows, cols, seed=rows + cols, spread=40.0)
    x[0, :16] = 0.0
    codes, scales = crisp.quantize(x.to(DEV))
    want_codes, want_scales = ref.quantize(f64(x))
    np.testing.assert_array_equal(raw(scales), want_scales)
    np.testing.assert_array_equal(raw(codes), want_codes)


def test_quantize_borders():
    """Magnitudes at the largest code and just above it, zeros, subnormals, the largest bf16 numbers, infinities and NaN."""
    x = torch.zeros(9, 256, dtype=torch.bfloat16)
    x[0, 3], x[0, 130] = 448.0, 450.0
    x[1, :128] = torch.linspace(-448, 448, 128).bfloat16()
    x[2, 0], x[2, 200] = 2.0 ** -133, -(2.0 ** -126)
    x[3, :] = torch.finfo(torch.bfloat16).max
    x[4, 5], x[4, 6], x[4, 7] = float("inf"), -float("inf"), 3.0
    x[5, 5], x[5, 6] = float("nan"), -2.0
    x[6, :] = float("inf")
    x[7, :] = float("nan")
    x[8, 128:] = 17.0 * 2.0 ** -100
    codes, scales = crisp.quantize(x.to(DEV))
    want_codes, want_scales = ref.quantize(f64(x))
    np.testing.assert_array_equal(raw(scales), want_scales)
    nan = np.isnan(f64(x))
    np.testing.assert_array_equal(raw(codes)[~nan], want_codes[~nan])
    assert ((raw(codes)[nan] & 0x7f) == 0x7f).all()


@pytest.mark.parametrize("rows,cols", [(1, (1 << 27) - 512), (5, 1 << 27), (3, (1 << 27) + 16), (1, (1 << 28) - 16), (2, 1 << 28)])
def test_quantize_widest(rows, cols):
    """Rows of up to 2^28 columns: each block of 128 is what it is in a row of its own, which the tests above pin."""
    base = normal(4096, 128, seed=11, spread=40.0).to(DEV)
    blocks = -(-cols // 128)
    x = torch.empty(rows, blocks * 128, dtype=torch.bfloat16, device=DEV)
    want_codes, want_scales = crisp.quantize(base)
    for r in range(rows):
        x[r] = base.roll(r, 0).repeat(-(-blocks // 4096), 1)[:blocks].view(-1)
    x = x[:, :cols].contiguous()
    codes, scales = crisp.quantize(x)
    del x
    for r in range(rows):
        whole = cols // 128
        part = lambda t: t.view(torch.uint8).roll(r, 0).repeat(-(-blocks // 4096), 1)[:blocks]  # noqa: E731
        assert torch.equal(codes[r].view(torch.uint8)[:whole * 128], part(want_codes)[:whole].view(-1))
        assert torch.equal(scales[r].view(torch.uint8)[:whole], part(want_scales[:, :1])[:whole, 0])
        if whole < blocks:
            last, scale = crisp.quantize(base.roll(r, 0)[whole % 4096, :cols % 128].view(1, -1).contiguous())
            assert torch.equal(codes[r].view(torch.uint8)[whole * 128:], last.view(torch.uint8)[0])
            assert scales[r].view(torch.uint8)[whole] == scale.view(torch.uint8)[0, 0]
        assert bool((scales[r].view(torch.uint8)[blocks:] == 127).all())


# ------------------------------------------------------------------------------------------------ norm
NORM_ERROR = 48 * 2.0 ** -24   # of y in fp32, relative: at most 32 + 15 roundings in the sum of squares (halved by the root),
#                                the division, the root (2 steps) and the two products


def check_norm(x, residual, weight, eps, quantized, **kw):
    y64, h64 = ref.norm(f64(x), None if residual is None else f64(residual), None if weight is None else f64(weight), eps)
    move = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    call = crisp.rms_norm_quantize if quantized else crisp.rms_norm
    *out, h = call(move(x), move(weight), move(residual), eps=eps, **kw)
    if residual is None:
        assert h is None
    else:
        np.testing.assert_array_equal(f64(h), h64)
    if not quantized:
        assert (np.abs(f64(out[0]) - y64) <= (HALF_BF16 + NORM_ERROR) * np.abs(y64) + 1e-38).all()
        return
    codes, scales = raw(out[0]), raw(out[1])
    blocks = -(-x.shape[1] // 128)
    assert (scales[:, blocks:] == 127).all()
    s = 2.0 ** (scales[:, :blocks].astype(np.float64) - 127)
    amax = np.stack([np.abs(y64[:, 128 * b:128 * b + 128]).max(1) for b in range(blocks)], 1)
    assert (amax <= 448 * s * (1 + NORM_ERROR)).all()
    assert ((amax > 224 * s * (1 - NORM_ERROR)) | (s == 2.0 ** -126)).all()
    full = np.repeat(s, 128, axis=1)[:, :x.shape[1]]
    # one rounding to the grid from a value within NORM_ERROR of y
    slack = NORM_ERROR * np.abs(y64)
    assert (np.abs(ref.values(codes, scales) - y64) <= ref.half_step((np.abs(y64) + slack) / full) * full + slack).all()


@pytest.mark.parametrize("cols", [16, 128, 240, 256, 272, 832, 1024, 1040, 2048, 3584, 4096, 4112, 8192, 16384, 16400, 32768])
@pytest.mark.parametrize("residual,quantized", [(True, True), (False, False), (True, False), (False, True)])
def test_norm(cols, residual, quantized):
    rows = 3 if cols > 4096 else 7
    x, r = normal(rows, cols, seed=cols, spread=6.0), normal(rows, cols, seed=cols + 1)
    w = (1 + 0.3 * normal(cols, seed=cols + 2).float()).bfloat16()
    check_norm(x, r if residual else None, w, 1e-5, quantized)


@pytest.mark.parametrize("rows,cols", [(1, 4096), (5000, 128), (3001, 1024)])
def test_norm_rows(rows, cols):
    """More rows than the GPU holds at a time, and one."""
    check_norm(normal(rows, cols, seed=3), normal(rows, cols, seed=4), None, 1e-6, True)


def test_norm_extremes():
    """Rows of zeros (eps alone), of tiny and of huge values; no eps."""
    x = normal(4, 512, seed=5)
    x[0], x[1], x[2] = 0.0, x[1] * 2.0 ** -60, x[2] * 2.0 ** 40
    for quantized in (False, True):
        check_norm(x, None, None, 1e-5, quantized)
        check_norm(x[1:], torch.zeros_like(x[1:]), None, 0.0, quantized)


@pytest.mark.parametrize("cols", [16, 512, 1024, 2048, 4096, 8192, 16384, 32768])
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-30])
@pytest.mark.parametrize("residual,quantized", [(True, True), (True, False), (False, True), (False, False)])
def test_norm_of_tiny_rows(cols, eps, residual, quantized):
    """Rows whose squares are near fp32's smallest number or below it, down to bf16's smallest, beside others."""
    x = normal(10, cols, seed=cols)
    for i, e in enumerate((0, -40, -48, -52, -60, -70, -80, -100, -126, -131)):
        x[i] = x[i] * 2.0 ** e
    w = (1 + 0.3 * normal(cols, seed=cols + 2).float()).bfloat16()
    check_norm(x, torch.zeros_like(x) if residual else None, w, eps, quantized)


@pytest.mark.parametrize("cols,rows", [(256, 5000), (1024, 3000), (4096, 1500), (16384, 400)])
def test_norm_of_many_tiny_rows(cols, rows):
    """More rows than are resident at a time, tiny ones and others in turn; over themselves too."""
    x = normal(rows, cols, seed=rows)
    x[::3], x[1::3] = x[::3] * 2.0 ** -120, x[1::3] * 2.0 ** -61
    check_norm(x, None, None, 0.0, False)
    check_norm(x, normal(rows, cols, seed=1) * 2.0 ** -75, None, 0.0, True)
    want, _ = crisp.rms_norm(x.to(DEV), eps=0.0)
    from paper_2609_01925_b200 import binding as B
    y = x.to(DEV)
    B.check(B.crisp_rms_norm(y, None, None, 0.0, None, y, None, None), "crisp_rms_norm")
    assert torch.equal(y, want)


def test_norm_of_zeros_without_eps():
    """0 / 0 is NaN, in its row alone."""
    x = normal(5, 512, seed=9)
    x[2] = 0.0
    y = f64(crisp.rms_norm(x.to(DEV), eps=0.0)[0])
    assert np.isnan(y[2]).all() and np.isfinite(np.delete(y, 2, 0)).all()
    assert (f64(crisp.rms_norm(x.to(DEV), eps=1e-40)[0])[2] == 0).all()


@pytest.mark.parametrize("cols", [80, 128, 4096])
def test_norm_at_the_bound_of_a_scale(cols):
    """Rows whose largest result is 448 * 2^-8 but for the roundings, and the 16-bit numbers beside it."""
    x = torch.stack([torch.full((cols,), c) for c in (0.3, 1.0, 7.0, 1e-3, 2.0 ** 30)]).bfloat16()
    for w in (1.75, 1.75 - 2.0 ** -7, 1.75 + 2.0 ** -7):
        check_norm(x, x * 0.7, torch.full((cols,), w).bfloat16(), 0.0, True)


def test_norm_nan_stays_in_its_row():
    x = normal(3, 4096, seed=6)
    clean = crisp.rms_norm_quantize(x.to(DEV))
    x[1, 77] = float("nan")
    codes, scales, _ = crisp.rms_norm_quantize(x.to(DEV))
    assert torch.equal(codes.view(torch.uint8)[::2], clean[0].view(torch.uint8)[::2])
    assert ((raw(codes)[1] & 0x7f) == 0x7f).all()


@pytest.mark.parametrize("into", ["x", "residual"])
def test_norm_sum_in_place(into):
    x, r = normal(600, 3584, seed=7).to(DEV), normal(600, 3584, seed=8).to(DEV)
    codes, scales, h = crisp.rms_norm_quantize(x, None, r)
    target = {"x": x, "residual": r}[into]
    codes2, scales2, h2 = crisp.rms_norm_quantize(x, None, r, sum_out=target)
    assert h2 is target and torch.equal(h, h2) and torch.equal(raw_t(codes), raw_t(codes2)) and torch.equal(raw_t(scales), raw_t(scales2))


def raw_t(t):
    return t.view(torch.uint8)


def test_norm_output_in_place():
    x, w = normal(700, 2048, seed=12).to(DEV), normal(2048, seed=13).to(DEV)
    want, _ = crisp.rms_norm(x, w)
    from paper_2609_01925_b200 import binding as B
    B.check(B.crisp_rms_norm(x, None, w, 1e-5, None, x, None, None), "crisp_rms_norm")
    assert torch.equal(x, want)


def test_norm_of_a_row_and_itself():
    """x as its own residual, stored over itself."""
    x = normal(300, 512, seed=14).to(DEV)
    want, h = crisp.rms_norm(x, None, x.clone())
    y, h2 = crisp.rms_norm(x, None, x, sum_out=x)
    assert torch.equal(y, want) and torch.equal(h2, h) and h2 is x


def test_norm_beyond_fp32():
    """Squares that leave fp32 make the row 0; the rows beside it are as they are."""
    x = normal(3, 1024, seed=15)
    x[1] = 2.0 ** 100
    y = f64(crisp.rms_norm(x.to(DEV))[0])
    assert (y[1] == 0).all()
    check_norm(x[::2].contiguous(), None, None, 1e-5, False)


def test_norm_of_a_stored_sum_is_the_same():
    x, r, w = normal(50, 4096, seed=9).to(DEV), normal(50, 4096, seed=10).to(DEV), normal(4096, seed=11).to(DEV)
    y, h = crisp.rms_norm(x, w, r)
    assert torch.equal(y, crisp.rms_norm(h, w)[0])


# ------------------------------------------------------------------------------------------------ product
def operand(rows, cols, seed, spread=8.0):
    x = normal(rows, cols, seed=seed, spread=spread)
    x[:, ::31] *= 6.0
    codes, scales = ref.quantize(f64(x))
    return codes, scales


def on_gpu(codes, scales):
    return (torch.from_numpy(codes).to(DEV).view(torch.float8_e4m3fn), torch.from_numpy(scales).to(DEV).view(torch.float8_e8m0fnu))


def check_product(a, w):
    lin = crisp.CrispLinear(*on_gpu(*w))
    out = lin(*on_gpu(*a))
    lin.poll()
    av, wv = (torch.from_numpy(ref.values(*t)).to(DEV) for t in (a, w))
    cols = av.shape[1]
    want = torch.zeros(av.shape[0], wv.shape[0], dtype=torch.float64, device=DEV)
    most = torch.zeros_like(want)
    for k in range(0, cols, 32):     # the largest sum on the way
        want += av[:, k:k + 32] @ wv[:, k:k + 32].t()
        most = torch.maximum(most, want.abs())
    most = torch.maximum(most, torch.minimum(av.abs().amax(1)[:, None] * wv.abs().amax(1)[None], (av.abs() @ wv.abs().t())))
    # bf16 once; each step of 32 columns adds 33 terms that are cut to 24 bits of the largest of them
    bound = HALF_BF16 * want.abs() + (cols // 32 + 1) * 33 * 2.0 ** -24 * most
    off = (out.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound.clamp(min=1e-300)).max())


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 100, 128, 129, 200, 255, 256, 257, 600])
@pytest.mark.parametrize("n,cols", [(128, 128), (256, 512), (130, 640), (1, 16), (77, 1040), (768, 2048)])
def test_product(rows, n, cols):
    check_product(operand(rows, cols, rows * 3 + cols), operand(n, cols, n * 7 + cols + 1))


@pytest.mark.parametrize("rows,n,cols", [(1, 6144, 4096), (33, 4096, 4096), (700, 4608, 3584), (3000, 1000, 1008), (64, 300, 16384),
                                         (5, 8192, 8192)])
def test_product_larger(rows, n, cols):
    check_product(operand(rows, cols, 1), operand(n, cols, 2))


@pytest.mark.parametrize("rows,n,cols", [(16, 128, 128), (256, 128, 512), (300, 260, 1168), (40, 1024, 4096), (1000, 700, 2064)])
def test_product_of_whole_numbers_is_exact(rows, n, cols):
    """Small whole numbers and scales between 2^-2 and 2^2, another one for every row and block: all sums are exact in fp32,
    so that a scale at the wrong row or block shows."""
    g = np.random.RandomState(rows + n + cols)
    grid = np.array([0x00, 0x38, 0x40, 0xb8, 0xc0], np.uint8)   # 0, 1, 2, -1, -2

    def make(r):
        codes, scales = grid[g.randint(0, 5, (r, cols))], np.full((r, ref.scale_cols(cols)), 127, np.uint8)
        scales[:, :-(-cols // 128)] = g.randint(125, 130, (r, -(-cols // 128)))
        return codes, scales

    a, w = make(rows), make(n)
    lin = crisp.CrispLinear(*on_gpu(*w))
    out = lin(*on_gpu(*a))
    lin.poll()
    want = torch.from_numpy(ref.values(*a)).to(DEV) @ torch.from_numpy(ref.values(*w)).to(DEV).t()
    assert torch.equal(out, want.bfloat16())      # |sums| < 2^24 / 16: exact in fp32, one rounding to bf16


@pytest.mark.parametrize("rows,n,cols", [(9000, 2056, 656), (9000, 2051, 656), (9000, 2050, 112), (2500, 4097, 1280), (20000, 45, 256),
                                         (3987, 20, 1120), (129, 6144, 2064), (1000, 1024, 8192), (48, 128, 20000), (200, 4224, 1024),
                                         (208, 2048, 2048), (230, 1000, 4096), (160, 512, 8192), (64, 20000, 512)])
def test_product_over_many_tiles_is_exact(rows, n, cols):
    """Several tiles one after the other in a CTA, rows of every alignment, few features, many columns: made on the GPU, otherwise
    as above."""
    g = torch.Generator(device=DEV).manual_seed(rows + n + cols)
    grid = torch.tensor([0x00, 0x38, 0x40, 0xb8, 0xc0], dtype=torch.uint8, device=DEV)
    number = torch.tensor([0.0, 1.0, 2.0, -1.0, -2.0], dtype=torch.float64, device=DEV)

    def make(r):
        pick = torch.randint(0, 5, (r, cols), generator=g, device=DEV)
        e = torch.randint(125, 130, (r, -(-cols // 128)), generator=g, device=DEV)
        scales = torch.full((r, ref.scale_cols(cols)), 127, dtype=torch.uint8, device=DEV)
        scales[:, :e.shape[1]] = e.to(torch.uint8)
        value = number[pick] * torch.exp2(e.double() - 127).repeat_interleave(128, 1)[:, :cols]
        return (grid[pick].view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)), value

    (a, av), (w, wv) = make(rows), make(n)
    lin = crisp.CrispLinear(*w)
    buffer = torch.full((rows + 3, n), 7.0, dtype=torch.bfloat16, device=DEV)
    lin(*a, out=buffer[:rows])
    lin.poll()
    assert torch.equal(buffer[:rows], (av @ wv.t()).bfloat16())
    assert bool((buffer[rows:] == 7.0).all())


@pytest.mark.parametrize("rows,n,cols", [(5, 130, 1 << 24), (300, 260, (1 << 22) + 16), (1, 1, 1 << 28)])
def test_product_of_very_many_columns(rows, n, cols):
    """Few elements of a row are not zero, the first and the last block's among them: exact."""
    g = torch.Generator(device=DEV).manual_seed(cols)
    at = torch.cat([torch.randint(0, cols, (400,), generator=g, device=DEV), torch.tensor([0, cols - 1, cols - 16], device=DEV)]).unique()
    grid = torch.tensor([0x38, 0x40, 0xb8], dtype=torch.uint8, device=DEV)         # 1, 2, -1
    number = torch.tensor([1.0, 2.0, -1.0], dtype=torch.float64, device=DEV)

    def make(r):
        pick = torch.randint(0, 3, (r, at.numel()), generator=g, device=DEV)
        codes = torch.zeros(r, cols, dtype=torch.uint8, device=DEV)
        codes[:, at] = grid[pick]
        scales = torch.full((r, ref.scale_cols(cols)), 127, dtype=torch.uint8, device=DEV)
        scales[:, ::3] = 128
        value = number[pick] * torch.where(at // 128 % 3 == 0, 2.0, 1.0).double()
        return (codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)), value

    (a, av), (w, wv) = make(rows), make(n)
    lin = crisp.CrispLinear(*w)
    out = lin(*a)
    lin.poll()
    assert torch.equal(out, (av @ wv.t()).bfloat16())


def test_product_extreme_scales_and_nan():
    """Scales whose products leave fp32 become 0 or infinity; a NaN code reaches its row of A, or its column, alone."""
    a, w = operand(20, 256, 3), operand(130, 256, 4)
    a[1][4], w[1][9] = 1, 1
    a[0][7, 100] = 0x7f
    w[0][50, 200] = 0xff
    out = f64(crisp.CrispLinear(*on_gpu(*w))(*on_gpu(*a)))
    nan = np.zeros((20, 130), bool)
    nan[7], nan[:, 50] = True, True
    assert (np.isnan(out) == nan).all()
    assert out[4, 9] == 0.0


def test_product_same_bits_again_and_beside_others():
    """The same call twice, and the same rows within a larger batch where the tiles are cut alike."""
    a, w = operand(33, 4096, 5), operand(4096, 4096, 6)
    lin = crisp.CrispLinear(*on_gpu(*w))
    one = lin(*on_gpu(*a))
    for _ in range(5):
        assert torch.equal(one, lin(*on_gpu(*a)))
    lin.poll()


def test_product_writes_its_rows_only():
    a, w = operand(30, 640, 7), operand(200, 640, 8)
    lin = crisp.CrispLinear(*on_gpu(*w))
    buffer = torch.full((40, 200), 7.0, dtype=torch.bfloat16, device=DEV)
    out = lin(*on_gpu(*a), out=buffer[:30])
    assert out.data_ptr() == buffer.data_ptr() and bool((buffer[30:] == 7.0).all())


# ------------------------------------------------------------------------------------------------ rotary
SCALINGS = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0, original=8192),
            dict(scaling="ramp", factor=8.0, original=8192), dict(scaling="bands", factor=8.0, original=8192),
            dict(scaling="ramp", factor=2.0, original=300, low=2.0, high=9.0), dict(scaling="bands", factor=16.0, original=100, low=0.5, high=3.0)]


def check_rotated(got, x, positions, freq, layout, magnitude):
    want = ref.rotate(x, positions, freq, layout, magnitude)
    size = np.zeros_like(want)
    n = len(freq)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + n)
        size[:, :, a] = size[:, :, b] = np.abs(x[:, :, a]) + np.abs(x[:, :, b])
    # bf16 once; the angle to 2^-25 turns (2e-7), cosine, sine and four products to 2^-22 together; the frequency itself, a
    # float64, to 2^-50 relative
    angle = 2e-7 + 2.0 ** -50 * np.abs(np.array([float(p) for p in positions]))[:, None, None]
    bound = HALF_BF16 * np.abs(want) + size * magnitude * (angle + 2.0 ** -22) + 1e-40
    assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim", [16, 48, 64, 112, 128])
@pytest.mark.parametrize("hq,hkv,n", [(4, 1, 1), (32, 8, 5), (6, 2, 700), (80, 8, 3)])
def test_rotary_split(layout, dim, hq, hkv, n):
    qkv = normal(n, (hq + 2 * hkv) * 128, seed=n + dim)
    positions = torch.randint(0, 1 << 20, (n,), generator=torch.Generator().manual_seed(n)).int()
    rot = crisp.CrispRotary(500000.0, rotary_dim=dim, layout=layout)
    q, k, v = rot.split(qkv.to(DEV), hq, hkv, positions.to(DEV))
    x = f64(qkv).reshape(n, -1, 128)
    freq = ref.frequencies(dim, 500000.0)
    check_rotated(f64(q), x[:, :hq], positions.tolist(), freq, layout, 1.0)
    check_rotated(f64(k), x[:, hq:hq + hkv], positions.tolist(), freq, layout, 1.0)
    np.testing.assert_array_equal(f64(v), x[:, hq + hkv:])
    np.testing.assert_array_equal(f64(q)[:, :, dim:], x[:, :hq, dim:])


@pytest.mark.parametrize("kw", SCALINGS)
@pytest.mark.parametrize("dim", [32, 128])
def test_rotary_scalings(kw, dim):
    x = normal(40, 3, 128, seed=dim)
    positions = [0, 1, 5, 8191, 8192, 131071, (1 << 31) - 1, -1, -(1 << 31)] + [(977 * i) % 100000 for i in range(31)]
    rot = crisp.CrispRotary(10000.0, rotary_dim=dim, **kw)
    magnitude = 0.1 * np.log(kw["factor"]) + 1.0 if kw.get("scaling") == "ramp" else 1.0
    assert abs(rot.plan.magnitude - magnitude) <= 1e-7 * magnitude
    got = rot.rotate(x.to(DEV), torch.tensor(positions, dtype=torch.int32, device=DEV))
    check_rotated(f64(got), f64(x), positions, ref.frequencies(dim, 10000.0, **kw), "half", magnitude)


def test_rotary_positions_in_order_and_strides():
    """Without positions the tokens count up from first_position; a slice of a wider tensor gives what its copy gives, also
    in place."""
    wide = normal(900, 10 * 128, seed=2).to(DEV)
    rot = crisp.CrispRotary(10000.0, layout="interleaved", rotary_dim=96)
    part = wide[:, 256:768].unflatten(1, (4, 128))
    positions = torch.arange(7000, 7900, dtype=torch.int32, device=DEV)
    a, b = rot.rotate(part, first_position=7000), rot.rotate(part.contiguous(), positions)
    assert torch.equal(a, b)
    own = part.contiguous()
    assert rot.rotate(own, positions, out=own) is own and torch.equal(own, a)
    q, k, v = rot.split(wide[:, 256:256 + 8 * 128], 4, 2, positions)
    assert torch.equal(q, a) and torch.equal(v, wide[:, 1024:1280].unflatten(1, (2, 128)))


def test_rotary_turns_back():
    x = normal(300, 8, 128, seed=3).to(DEV)
    positions = torch.randint(1, 1 << 30, (300,)).int().to(DEV)
    rot = crisp.CrispRotary(10000.0)
    back = rot.rotate(rot.rotate(x, positions), -positions)
    # two roundings to bf16, the first of which the way back spreads over the pair
    size = (x.float()[..., :64] ** 2 + x.float()[..., 64:] ** 2).sqrt().repeat(1, 1, 2)
    assert bool(((back.float() - x.float()).abs() <= size * (2.5 * HALF_BF16)).all())


# ------------------------------------------------------------------------------------------------ large tensors
def test_offsets_beyond_32_bits():
    """Tensors of more than 2^31 elements: their last rows, and those around element 2^31, are what the same rows give alone."""
    rows, cols = 530000, 4096
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    base = torch.randn(1000, cols, generator=g, device=DEV).bfloat16()
    for at in range(0, rows, 1000):
        x[at:at + 1000] = base.roll(at // 1000, 0)
    parts = [slice(0, 3), slice(2 ** 31 // cols - 2, 2 ** 31 // cols + 3), slice(rows - 5, rows)]
    residual = x.flip(0)
    codes, scales, h = crisp.rms_norm_quantize(x, None, residual)
    qc, qs = crisp.quantize(x)
    for p in parts:
        a = crisp.rms_norm_quantize(x[p].contiguous(), None, residual[p].contiguous())
        assert torch.equal(raw_t(codes[p]), raw_t(a[0])) and torch.equal(raw_t(scales[p]), raw_t(a[1])) and torch.equal(h[p], a[2])
        b = crisp.quantize(x[p].contiguous())
        assert torch.equal(raw_t(qc[p]), raw_t(b[0])) and torch.equal(raw_t(qs[p]), raw_t(b[1]))
    del residual, codes, scales, h, qc, qs, x
    rows, n = 360000, 6144
    a = crisp.quantize(torch.randn(rows, 128, generator=g, device=DEV).bfloat16())
    lin = crisp.CrispLinear.from_weight(torch.randn(n, 128, generator=g, device=DEV).bfloat16())
    out = lin(*a)
    rot = crisp.CrispRotary(1e4)
    q, k, v = rot.split(out, 32, 8)
    parts = [slice(0, 300), slice(2 ** 31 // n - 150, 2 ** 31 // n + 150), slice(rows - 300, rows)]
    for p in parts:
        want = lin(*(t[p].contiguous() for t in a))
        # (another cut of the product: sums of 128 columns in one order, so the same bits)
        assert torch.equal(out[p], want)
        again = rot.split(want, 32, 8, torch.arange(p.start, p.stop, dtype=torch.int32, device=DEV))
        assert all(torch.equal(s[p], t) for s, t in zip((q, k, v), again))
    lin.poll()


# ------------------------------------------------------------------------------------------------ sizes of zero, refusals
def test_nothing_to_do():
    empty = torch.empty(0, 256, dtype=torch.bfloat16, device=DEV)
    codes, scales = crisp.quantize(empty)
    assert codes.shape == (0, 256) and scales.shape == (0, 4)
    y, h = crisp.rms_norm(empty, None, empty)
    assert y.shape == h.shape == (0, 256)
    lin = crisp.CrispLinear(*crisp.quantize(normal(32, 256).to(DEV)))
    assert lin(codes, scales).shape == (0, 32)
    rot = crisp.CrispRotary(10000.0)
    q, k, v = rot.split(empty[:, :0].expand(0, 0).reshape(0, 0).new_empty(0, 4 * 128), 2, 1)
    assert q.shape == (0, 2, 128) and v.shape == (0, 1, 128)
    assert rot.rotate(torch.empty(0, 2, 128, dtype=torch.bfloat16, device=DEV)).shape == (0, 2, 128)


def test_refusals():
    x = normal(4, 256).to(DEV)
    codes, scales = crisp.quantize(x)
    lin = crisp.CrispLinear(codes, scales)
    for bad in (lambda: crisp.quantize(x.float()), lambda: crisp.quantize(x[:, ::2]), lambda: crisp.quantize(x[0]),
                lambda: crisp.rms_norm(x, x[0, :128]), lambda: crisp.rms_norm(x, None, x[:2]), lambda: crisp.rms_norm(x, sum_out=x),
                lambda: crisp.rms_norm(x, None, x, sum_out=x[:2]), lambda: crisp.CrispLinear(codes, scales[:, :2]),
                lambda: crisp.CrispLinear(codes.view(torch.uint8), scales), lambda: lin(codes[:, :128].contiguous(), scales),
                lambda: lin(codes, scales[:2]), lambda: lin(codes, scales, out=x),
                lambda: crisp.CrispRotary(1e4).split(x, 1, 1), lambda: crisp.CrispRotary(1e4).rotate(x)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: crisp.quantize(normal(4, 24).to(DEV)), lambda: crisp.rms_norm(normal(1, 32784).to(DEV)),
                lambda: crisp.rms_norm(x, eps=-1.0), lambda: crisp.rms_norm(x, eps=float("nan"))):
        with pytest.raises(crisp.CrispError):
            bad()
