"""The 8-bit decoder operators on the GPU against their definitions in 64 bits.

Tolerances, from the number formats: half a unit in the last place of an output
(E4M3 2^-4, bfloat16 2^-8, float16 2^-11, float32 2^-24, relative), and the terms'
own errors: 2^-23 a step for sums in 32 bits, 2^-13 of a block's largest products for
the 8-bit matrix instruction, 2^-11 for softmax weights held as 16-bit floats.
Quantisers without a gate and the cache are exact: their bytes are compared.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
HALF_ULP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF16: 2.0 ** -133, F16: 2.0 ** -25, F32: 2.0 ** -149}


@pytest.fixture(scope="module")
def ops():
    from paper_1905_13298_amd import ops as o
    return o


def normal(seed, *shape, std=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std


def least_byte(amax):
    """The scale byte of each block from its largest magnitude, in 64 bits."""
    amax = amax.double()
    e = torch.ceil(torch.log2(torch.where(amax > 0, amax, 448.0) / 448.0))
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, e)
    e = torch.where(amax <= 448.0 * torch.exp2(e - 1), e - 1, e)
    return torch.where(amax > 0, (e + 127).clamp(1, 254), 127.0).long()


def blocks(y, rows=1):
    r, c = y.shape
    y = torch.nn.functional.pad(y, (0, -c % 128, 0, -r % rows))
    return y.reshape(y.shape[0] // rows, rows, y.shape[1] // 128, 128)


def spread(e, like, rows=1):
    """A block's value for each of its elements."""
    r, c = like.shape
    return e.repeat_interleave(rows, 0)[:r].repeat_interleave(128, 1)[:, :c]


def value(q, scales, rows=1):
    e = spread(scales.cpu().view(torch.uint8).long(), q, rows)
    return q.cpu().double() * torch.exp2((e - 127).double())


def to8(y, rows=1):
    """(E4M3 numbers, scale bytes) of y by the definition (exact for float32 inputs)."""
    b = blocks(y.float(), rows)
    e = least_byte(torch.where(torch.isfinite(b), b.abs(), 0.0).amax((1, 3)))
    q = (y.double() * torch.exp2(-(spread(e, y, rows) - 127).double())).float()
    return q.to(E4M3), e.to(torch.uint8)


def same_bytes(a, b):
    a, b = a.cpu().view(torch.uint8), b.cpu().view(torch.uint8)
    nan = (a & 0x7F) == 0x7F
    return torch.equal(nan, (b & 0x7F) == 0x7F) and torch.equal(a[~nan], b[~nan])


def near8(q, scales, y, slack):
    """8-bit numbers of a computed y: each within half a unit of y (that is off by `slack`, relative),
    each scale the least possible or, at a boundary within the slack, its neighbour."""
    e = scales.cpu().view(torch.uint8).long()
    amax = blocks(y).abs().amax((1, 3))
    assert torch.all((e >= least_byte(amax * (1 - slack))) & (e <= least_byte(amax * (1 + slack))))
    got, step = value(q, scales), torch.exp2((spread(e, y) - 127).double())
    tol = torch.maximum(y.abs() * 2.0 ** -4, step * 2.0 ** -10) + y.abs() * slack * 2
    assert torch.all((got - y).abs() <= tol)


def same(a, b):
    return a.shape == b.shape and a.dtype == b.dtype and bool(torch.equal(a, b))


def near(got, want, terms=0.0):
    """got within its type's rounding of `want` and of what the terms are off by."""
    t = got.dtype
    assert torch.isfinite(got).all()
    off = (got.cpu().double() - want).abs()
    tol = want.abs() * HALF_ULP[t] * 1.01 + TINY[t] + terms * (1 + HALF_ULP[t])
    assert torch.all(off <= tol), float((off / tol.clamp(min=1e-300)).max())


# ---------------------------------------------------------------------------
# Norm.

def rms(x, w, r, eps, dtype):
    h = x.double() if r is None else (x.float() + r.float()).to(dtype).double()
    rstd = (h.square().mean(1) + eps).rsqrt()
    return h, rstd, h * rstd[:, None] * w.double()


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 128), (5, 129), (4, 512), (7, 1000), (3, 1024), (3, 1025), (2, 2049),
                                       (9, 4096), (2, 8200), (1, 16385), (1, 40000), (300, 96)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_norm(ops, rows, cols, dtype):
    x, r, w = normal(1, rows, cols).to(dtype), normal(2, rows, cols, std=3).to(dtype), (normal(3, cols, std=0.2) + 1).to(dtype)
    slack = 1e-5 + cols * 2.0 ** -24
    for res in (None, r):
        for quantize in (True, False):
            y, s, h, rstd = ops.rms_norm(x.to(DEV), w.to(DEV), None if res is None else res.to(DEV), eps=1e-5, quantize=quantize)
            hw, rw, yw = rms(x, w, res, 1e-5, dtype)
            assert torch.equal(h.cpu().double(), hw)
            assert torch.all((rstd.cpu().double() - rw).abs() <= rw * slack)
            assert y.shape == (rows, cols)
            if quantize:
                assert y.dtype == E4M3 and s.dtype == E8M0 and s.shape == (rows, (cols + 127) // 128)
                near8(y, s, yw, slack)
            else:
                assert s is None
                near(y, yw, yw.abs() * slack)


def test_norm_strides_weight_type_and_special_rows(ops):
    x = normal(4, 6, 300).to(BF16)
    x[1] = 0
    x[2, 5] = float("inf")
    x[3, 6] = float("nan")
    wide = torch.zeros(6, 999, dtype=BF16)
    wide[:, 17:317] = x
    w = normal(5, 300) + 1
    y, s, h, rstd = ops.rms_norm(wide.to(DEV)[:, 17:317], w.to(DEV), quantize=True)
    _, rw, yw = rms(x, w, None, 1e-6, BF16)
    keep = [0, 1, 4, 5]
    assert torch.allclose(rstd.cpu().double()[keep], rw[keep], rtol=1e-5)
    near8(y[keep], s.view(torch.uint8)[keep], yw[keep], 1e-4)
    assert torch.all(value(y, s)[1] == 0)
    # An infinite element makes the norm 0 and itself 0 * inf; a NaN makes the whole row NaN.
    assert math.isnan(float(value(y, s)[2, 5])) and float(value(y, s)[2].nan_to_num().abs().max()) == 0
    assert torch.isnan(value(y, s)[3]).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 129), (7, 1000), (5, 1024), (600, 64), (9, 2050), (3, 4096), (520, 4100), (1, 20000)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_norm_gradient(ops, rows, cols, dtype):
    h, w, dy, dh = (normal(i, rows, cols).to(dtype) for i in range(4))
    w = (w[0] * 0.2 + 1).to(dtype)
    rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
    hd, wd, dyd, rd = h.double(), w.double(), dy.double(), rstd.double()[:, None]
    n, g = hd * rd, dyd * wd
    inner = (g * n).mean(1, keepdim=True)
    dx = rd * (g - n * inner)
    size = rd * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True)) * (cols * 2.0 ** -24 + 2.0 ** -20)
    dw, dsize = (dyd * n).sum(0), (dyd * n).abs().sum(0) * (rows * 2.0 ** -24 + 2.0 ** -20)
    for extra in (None, dh):
        got, gw = ops.rms_norm_backward(dy.to(DEV), h.to(DEV), w.to(DEV), rstd.to(DEV), None if extra is None else extra.to(DEV))
        want = dx if extra is None else dx + dh.double()
        near(got, want, size + want.abs() * 2.0 ** -22)
        near(gw, dw, dsize)
    again = ops.rms_norm_backward(dy.to(DEV), h.to(DEV), w.to(DEV), rstd.to(DEV), dh.to(DEV))
    assert torch.equal(again[0], got) and torch.equal(again[1], gw)


def test_norm_gradient_against_differences(ops):
    """Central differences of the float32 norm: sum(y * c) for random c, along random directions."""
    rows, cols = 3, 160
    x, w, c = normal(1, rows, cols), normal(2, cols, std=0.2) + 1, normal(3, rows, cols)
    loss = lambda x, w: float((rms(x, w, None, 1e-6, F32)[2] * c.double()).sum())  # noqa: E731
    _, _, h, rstd = ops.rms_norm(x.to(DEV), w.to(DEV), quantize=False)
    dx, dw = ops.rms_norm_backward(c.to(DEV), h, w.to(DEV), rstd)
    for seed in range(5):
        u, v = normal(10 + seed, rows, cols).double(), normal(20 + seed, cols).double()
        t = 1e-4
        num = (loss(x.double() + t * u, w.double() + t * v) - loss(x.double() - t * u, w.double() - t * v)) / (2 * t)
        ana = float((dx.cpu().double() * u).sum() + (dw.cpu().double() * v).sum())
        # t^2 times a third derivative of order sum |c| for the differences, 2^-20 a term for the gradients.
        assert abs(num - ana) <= 1e-5 * float((dx.cpu().double() * u).abs().sum() + (dw.cpu().double() * v).abs().sum())


def test_norm_gradient_strides_weight_type_and_no_rows(ops):
    rows, cols = 5, 333
    big = normal(1, 3, rows, 2 * cols)
    dy, h, dh = (big[i, :, i:i + cols] for i in range(3))
    w, rstd = normal(2, cols) + 1, torch.rand(rows, generator=torch.Generator().manual_seed(1)) + 0.5
    d = big.to(BF16).to(DEV)
    got, gw = ops.rms_norm_backward(*(d[i, :, i:i + cols] for i in (0, 1)), w.to(DEV), rstd.to(DEV), d[2, :, 2:2 + cols])
    assert gw.dtype == F32
    same, sw = ops.rms_norm_backward(dy.to(BF16).to(DEV).contiguous(), h.to(BF16).to(DEV).contiguous(), w.to(DEV), rstd.to(DEV),
                                     dh.to(BF16).to(DEV).contiguous())
    assert torch.equal(got, same) and torch.equal(gw, sw)
    none = torch.empty(0, cols, dtype=BF16, device=DEV)
    dx, dw = ops.rms_norm_backward(none, none, w.to(DEV), torch.empty(0, device=DEV))
    assert dx.shape == (0, cols) and torch.all(dw == 0)
    assert ops.rms_norm(none, w.to(DEV))[0].shape == (0, cols)


# ---------------------------------------------------------------------------
# Quantisers.

@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 5), (2, 127), (2, 128), (4, 129), (5, 1000), (33, 4096), (257, 40)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_quantize(ops, rows, cols, dtype):
    x = (normal(rows, rows, cols) * torch.exp2(normal(2, rows, 1) * 4)).to(dtype)
    q, s = ops.quantize_fp8(x.to(DEV))
    qw, ew = to8(x)
    assert same_bytes(s, ew) and same_bytes(q, qw)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 200), (40, 1000), (5, 4096)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_quantize_with_gate(ops, rows, cols, dtype):
    both = normal(7, rows, 2 * cols + 3, std=3).to(dtype)
    g, x = both[:, :cols], both[:, cols + 3:]
    d = both.to(DEV)
    q, s = ops.quantize_fp8(d[:, cols + 3:], d[:, :cols])
    y = x.double() * g.double() * torch.sigmoid(g.double())
    near8(q, s, y, 1e-5)


def test_quantize_boundaries_and_special_values(ops):
    x = torch.zeros(9, 128)
    x[0, 0] = 448.0                                   # scale 1
    x[1, 0] = 448.00003                               # the next power
    x[2, :2] = torch.tensor([float("inf"), 3.0])
    x[3, :2] = torch.tensor([float("nan"), -7.0])
    x[4, 0] = 3.4e38
    x[5, 0] = 1e-45
    x[6, :3] = torch.tensor([2.0 ** -120, -2.0 ** -130, 0.0])
    x[7] = torch.linspace(-448, 448, 128)
    x[8] = float("-inf")
    q, s = ops.quantize_fp8(x.to(DEV))
    qw, ew = to8(x)
    assert same_bytes(s, ew) and same_bytes(q, qw)
    assert int(s.view(torch.uint8)[0, 0]) == 127 and int(s.view(torch.uint8)[1, 0]) == 128
    assert int(s.view(torch.uint8)[8, 0]) == 127


@pytest.mark.parametrize("rows,cols", [(1, 1), (127, 130), (128, 128), (300, 1000)])
def test_quantize_weights(ops, rows, cols):
    w = (normal(3, rows, cols) * torch.exp2(normal(4, rows, 1))).to(BF16)
    w8, s = ops.quantize_weights_fp8(w.to(DEV))
    qw, ew = to8(w, 128)
    assert same_bytes(s, ew) and same_bytes(w8, qw)


@pytest.mark.parametrize("bits", [2, 3, 4, 5])
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 37), (64, 512), (3, 4099)])
def test_shift_weights(ops, rows, cols, bits):
    rng = np.random.default_rng(rows + bits)
    sh = rng.integers(0, 2 ** (bits - 1) - 1, (rows, cols))
    codes = np.where(rng.random((rows, cols)) < 0.2, 15, sh) + 16 * rng.integers(0, 2, (rows, cols))
    codes = codes.astype(np.uint8)
    w8, s = ops.shift_weights_to_fp8(torch.from_numpy(ops.pack_shift_weights(codes, bits).view(np.int32)).to(DEV), cols, bits)
    want = np.where((codes & 15) == 15, 0.0, np.where(codes & 16, -1.0, 1.0) * 2.0 ** -(codes & 15).astype(float))
    assert np.array_equal(w8.cpu().double().numpy(), want)
    assert torch.all(s.cpu().float() == 1)


# ---------------------------------------------------------------------------
# Product.

def operands(ops, m, n, k, wtype, seed=0):
    x8, xs = ops.quantize_fp8((normal(seed, m, k) * torch.exp2(normal(seed + 1, m, 1))).to(DEV))
    if wtype == E4M3:
        w8, ws = ops.quantize_weights_fp8(normal(seed + 2, n, k, std=0.05).to(DEV))
    else:
        rng = np.random.default_rng(seed)
        codes = (rng.integers(0, 16, (n, k)) + 16 * rng.integers(0, 2, (n, k))).astype(np.uint8)
        w8, ws = ops.shift_weights_to_fp8(torch.from_numpy(ops.pack_shift_weights(codes).view(np.int32)).to(DEV), k)
    return x8, xs, w8, ws


def product_terms(x, w, k, full):
    """What the sums may be off by: a 32-bit rounding for each block of 32 or 128, and for the 8-bit instruction
    2^-13 of each block's largest product, which a row's largest stand above."""
    sums = x.abs() @ w.abs().T
    if full:
        return sums * (k / 32 + 3) * 2.0 ** -23
    per = sum(x[:, i:i + 128].abs().amax(1, keepdim=True) * w[:, i:i + 128].abs().amax(1)[None, :] for i in range(0, k, 128))
    return per * 2.0 ** -13 * 4 + sums * (k / 128 + 3) * 2.0 ** -23


SHAPES = [(1, 1, 1), (1, 16, 128), (3, 17, 129), (16, 64, 256), (17, 100, 1000), (5, 128, 4096), (33, 31, 15), (64, 256, 512),
          (65, 129, 640), (130, 260, 384), (256, 256, 128), (300, 500, 1100), (513, 300, 272), (1000, 1030, 160)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("wtype", [E4M3, E5M2])
@pytest.mark.parametrize("out", [BF16, F16, F32])
def test_product(ops, m, n, k, wtype, out):
    x8, xs, w8, ws = operands(ops, m, n, k, wtype, m + k)
    bias = normal(9, n)
    x, w = value(x8, xs), value(w8, ws, 128)
    terms = product_terms(x, w, k, out == F32)
    y = ops.linear_fp8(x8, xs, w8, ws, out_dtype=out)
    assert y.dtype == out and y.shape == (m, n)
    near(y, x @ w.T, terms)
    y = ops.linear_fp8(x8, xs, w8, ws, bias.to(DEV), out_dtype=out)
    near(y, x @ w.T + bias.double(), terms + (x @ w.T).abs() * 2.0 ** -23)


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("wtype", [E4M3, E5M2])
@pytest.mark.parametrize("out", [BF16, F32])
def test_product_input_gradient(ops, m, n, k, wtype, out):
    _, _, w8, ws = operands(ops, 1, n, k, wtype, m + k)
    dy8, ds = ops.quantize_fp8(normal(5, m, n, std=1e-3).to(DEV))
    dy, w = value(dy8, ds), value(w8, ws, 128)
    dx = ops.linear_fp8_backward_data(dy8, ds, w8, ws, out_dtype=out)
    near(dx, dy @ w, product_terms(dy, w.T.contiguous(), n, out == F32))


@pytest.mark.parametrize("m,n,k", [(20, 11000, 130), (50, 5501, 272), (1, 9000, 1100), (40, 130, 700), (700, 300, 640), (1000, 3000, 333), (2561, 4100, 1), (2561, 4100, 136), (4100, 2700, 250), (2561, 4100, 384),
                                   (2817, 3900, 655), (2561, 4100, 4230), (5000, 4400, 1000)])
@pytest.mark.parametrize("wtype,out", [(E4M3, BF16), (E5M2, F16)])
def test_product_of_many_tiles(ops, m, n, k, wtype, out):
    """Every tile's edges in the columns, the first and last rows and some between."""
    x8, xs, w8, ws = operands(ops, m, n, k, wtype, m + k)
    y = ops.linear_fp8(x8, xs, w8, ws, out_dtype=out).cpu()
    rows = torch.unique(torch.cat([torch.arange(min(m, 20)), torch.arange(max(m - 20, 0), m), torch.arange(0, m, 37)]))
    x, w = value(x8, xs)[rows], value(w8, ws, 128)
    near(y[rows], x @ w.T, product_terms(x, w, k, False))


def test_product_is_exact_on_small_integers_and_equals_linear_shift(ops):
    """Integers times signed powers of two: every sum is exact, so the 8-bit product equals LinearShift on inputs whose
    shifts lose nothing."""
    m, n, k = 70, 90, 300
    rng = np.random.default_rng(3)
    xi = rng.integers(-8, 9, (m, k))
    codes = (rng.integers(0, 5, (n, k)) + 16 * rng.integers(0, 2, (n, k))).astype(np.uint8)
    wp = torch.from_numpy(ops.pack_shift_weights(codes).view(np.int32)).to(DEV)
    want = ops.linear_shift(torch.from_numpy((xi * 2 ** 16).astype(np.int32)).to(DEV), wp).cpu().double() / 2 ** 16
    w8, ws = ops.shift_weights_to_fp8(wp, k)
    x8, xs = ops.quantize_fp8(torch.from_numpy(xi.astype(np.float32)).to(DEV))
    assert torch.equal(ops.linear_fp8(x8, xs, w8, ws, out_dtype=F32).cpu().double(), want)


def test_product_never_uses_what_lies_past_the_columns(ops):
    """NaN bytes and NaN scales behind a row's end change nothing; strided scales are read as they lie."""
    for m, n, k in ((20, 40, 100), (3, 20, 257), (300, 300, 330)):
        x8, xs, w8, ws = operands(ops, m, n, k, E4M3)
        want = ops.linear_fp8(x8, xs, w8, ws)
        wide = []
        for t in (x8, w8):
            b = torch.full((t.shape[0], (k + 15) // 16 * 16 + 64), 0x7F, dtype=torch.uint8, device=DEV).view(E4M3)
            b[:, 16:16 + k].copy_(t)
            wide.append(b[:, 16:16 + k])
        sc = []
        for t in (xs, ws):
            b = torch.full((t.shape[0], t.shape[1] + 5), 0xFF, dtype=torch.uint8, device=DEV)
            b[:, 1:1 + t.shape[1]] = t.view(torch.uint8)
            sc.append(b.view(E8M0)[:, 1:1 + t.shape[1]])
        assert torch.equal(ops.linear_fp8(wide[0], sc[0], wide[1], sc[1]), want)
        dy8, ds = ops.quantize_fp8(normal(1, m, n).to(DEV))
        assert torch.equal(ops.linear_fp8_backward_data(dy8, ds, wide[1], sc[1]), ops.linear_fp8_backward_data(dy8, ds, w8, ws))


def test_product_of_rows_that_are_not_on_16_bytes(ops):
    m, n, k = 9, 33, 101
    x8, xs, w8, ws = operands(ops, m, n, k, E4M3)
    want = ops.linear_fp8(x8, xs, w8, ws)
    assert torch.equal(ops.linear_fp8(x8.contiguous(), xs, w8.contiguous(), ws), want)


def test_product_special_values(ops):
    """A NaN reaches its own row (x) or column (w) of y alone, a NaN scale its block's; no tokens give no rows."""
    m, n, k = 40, 50, 256
    x8, xs, w8, ws = operands(ops, m, n, k, E4M3)
    want = ops.linear_fp8(x8, xs, w8, ws).cpu()
    x2, w2 = x8.clone(), w8.clone()
    x2.view(torch.uint8)[3, 200] = 0x7F
    w2.view(torch.uint8)[11, 7] = 0xFF
    got = ops.linear_fp8(x2, xs, w2, ws).cpu()
    nan = torch.zeros(m, n, dtype=torch.bool)
    nan[3], nan[:, 11] = True, True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])
    assert ops.linear_fp8(x8[:0], xs[:0], w8, ws).shape == (0, n)


def test_product_scales_at_the_ends_of_their_range(ops):
    """Scales of 2^-60 and 2^60 that cancel: the products' sizes are ordinary."""
    m, n, k = 20, 24, 384
    x8, xs, w8, ws = operands(ops, m, n, k, E4M3)
    for out in (BF16, F32):
        want = ops.linear_fp8(x8, xs, w8, ws, out_dtype=out)
        up, down = (xs.view(torch.uint8) + 60).view(E8M0), (ws.view(torch.uint8) - 60).view(E8M0)
        assert torch.equal(ops.linear_fp8(x8, up, w8, down, out_dtype=out), want)


# ---------------------------------------------------------------------------
# Cache.

def cache_scale(amax):
    e = least_byte(amax)
    return torch.where(amax > 0, e.clamp(127 - 48, 127 + 48), 127 - 48)


def append_reference(k8, ks, new, table, start, count, page, last):
    """One cache after the append, byte for byte: a loop over tokens' pages."""
    k8, ks = k8.cpu().clone(), ks.cpu().view(torch.uint8).clone()
    batch, tokens, heads, dim = new.shape
    for b in range(batch):
        s, n = int(start[b]), min(int(count[b]), tokens)
        for col in range(s // page, (s + n - 1) // page + 1) if n > 0 else ():
            if col >= table.shape[1] or not 0 <= int(table[b, col]) < k8.shape[0]:
                continue
            pid, lo, hi = int(table[b, col]), max(s - col * page, 0), min(s + n - col * page, page)
            for h in range(heads):
                x = new[b, col * page + lo - s:col * page + hi - s, h].float()
                e = int(cache_scale(torch.where(torch.isfinite(x), x.abs(), 0.0).max()))
                held = k8[pid, h].view(torch.uint8).T.contiguous().view(E4M3) if last else k8[pid, h]
                held = held.clone()
                if lo > 0:
                    before = min(max(int(ks[pid, h]), 79), 175)
                    if before > e:
                        e = before
                    held[:lo] = (held[:lo].float() * 2.0 ** (before - e)).to(E4M3)
                y = (x.double() * 2.0 ** -(e - 127)).float()
                held[lo:hi] = torch.where(torch.isfinite(x), y.clamp(-448, 448), math.nan).to(E4M3)
                k8[pid, h] = held.view(torch.uint8).T.contiguous().view(E4M3) if last else held
                ks[pid, h] = e
    return k8, ks


def filled_cache(ops, pages, heads, page, dim, seed=0):
    k8, v8, ks, vs = ops.kv_cache(pages, heads, page, dim, DEV)
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[:, None]
    k = normal(seed, pages, page, heads, dim) * torch.exp2(normal(seed + 1, pages, page, 1, 1))
    v = normal(seed + 2, pages, page, heads, dim) * torch.exp2(normal(seed + 3, pages, page, 1, 1))
    ops.kv_cache_append(k.to(DEV), v.to(DEV), k8, v8, ks, vs, table, torch.zeros(pages, dtype=torch.int32, device=DEV))
    return k8, v8, ks, vs


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dim,heads", [(16, 1), (64, 3), (80, 2), (128, 2), (256, 1)])
@pytest.mark.parametrize("tokens", [1, 5, 70, 150])
def test_append(ops, page, dim, heads, tokens):
    batch, columns = 5, (400 + page - 1) // page
    gen = torch.Generator().manual_seed(page + dim + tokens)
    pages = batch * columns + 2
    cache = filled_cache(ops, pages, heads, page, dim)
    table = torch.randperm(pages, generator=gen)[:batch * columns].reshape(batch, columns).to(torch.int32)
    start = torch.tensor([0, 1, page - 1, page, 211], dtype=torch.int32)
    count = torch.tensor([tokens, tokens, max(tokens - 1, 1), 0, tokens], dtype=torch.int32)
    dtype = (BF16, F16, F32)[dim % 3]
    big = normal(5, 2, batch, tokens, heads, dim + 3, std=2).to(dtype)
    k, v = (big[i, ..., i:i + dim] for i in range(2))
    want = [append_reference(cache[i], cache[2 + i], (k, v)[i], table, start, count, page, bool(i)) for i in range(2)]
    d = big.to(DEV)
    ops.kv_cache_append(d[0, ..., 0:dim], d[1, ..., 1:1 + dim], *cache, table.to(DEV), start.to(DEV), count.to(DEV))
    for i in range(2):
        assert same_bytes(cache[i], want[i][0])
        assert torch.equal(cache[2 + i].cpu().view(torch.uint8), want[i][1])


def test_append_drops_what_has_no_page_and_bounds_values(ops):
    page, dim, heads = 16, 32, 1
    cache = filled_cache(ops, 4, heads, page, dim)
    before = [t.cpu().view(torch.uint8).clone() for t in cache]
    table = torch.tensor([[-1, 3], [7, 0]], dtype=torch.int32)     # columns without a page, and past the table
    k = normal(1, 2, 40, heads, dim)
    k[0, 20, 0, 0], k[0, 21, 0, 1], k[0, 22, 0, 2] = 1e30, float("inf"), float("nan")
    k[1, 16:, 0] *= 1e-25                                           # below the least scale
    zero = torch.zeros(2, dtype=torch.int32)
    count = torch.full((2,), 40, dtype=torch.int32)
    want = [append_reference(cache[i], cache[2 + i], k, table, zero, count, page, bool(i)) for i in range(2)]
    ops.kv_cache_append(k.to(DEV), k.to(DEV), *cache, table.to(DEV), zero.to(DEV))
    for i in range(2):
        assert same_bytes(cache[i], want[i][0])
        assert torch.equal(cache[2 + i].cpu().view(torch.uint8), want[i][1])
        for p in (1, 2):
            assert torch.equal(cache[i].cpu().view(torch.uint8)[p], before[i][p])
    held = cache[0].cpu()[3, 0].float()
    assert held[4, 0] == 448 and torch.isnan(held[5, 1]) and torch.isnan(held[6, 2])


def test_append_one_by_one_grows_scales(ops):
    """Tokens of growing size into one page, one call each: byte for byte the definition's repeated rounding."""
    page, dim, heads = 32, 64, 2
    cache = ops.kv_cache(1, heads, page, dim, DEV)
    want = [(cache[i].cpu(), cache[2 + i].cpu().view(torch.uint8)) for i in range(2)]
    table, one = torch.zeros(1, 1, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    x = normal(3, 20, 1, 1, heads, dim) * torch.exp2(torch.arange(20).float() * 0.7)[:, None, None, None, None]
    for t in range(20):
        start = torch.tensor([t], dtype=torch.int32)
        want = [append_reference(want[i][0], want[i][1], x[t], table, start, one, page, bool(i)) for i in range(2)]
        ops.kv_cache_append(x[t].to(DEV), x[t].to(DEV), *cache, table.to(DEV), start.to(DEV))
    for i in range(2):
        assert same_bytes(cache[i], want[i][0])
        assert torch.equal(cache[2 + i].cpu().view(torch.uint8), want[i][1])


# ---------------------------------------------------------------------------
# Attention.

def attention_reference(q, cache, table, length, count, window, scale):
    """(o, what it may be off by) in 64 bits, a query head at a time."""
    k8, v8, ks, vs = (t.cpu() for t in cache)
    pages, heads, page, dim = k8.shape
    kv = k8.double() * torch.exp2(ks.view(torch.uint8).double() - 127)[:, :, None, None]
    vv = (v8.double() * torch.exp2(vs.view(torch.uint8).double() - 127)[:, :, None, None]).transpose(2, 3)
    batch, tokens, hq, _ = q.shape
    group = hq // heads
    o, off = torch.zeros(batch, tokens, hq, dim, dtype=torch.float64), torch.zeros(batch, tokens, hq, dim, dtype=torch.float64)
    for b in range(batch):
        n = min(max(int(length[b]), 0), table.shape[1] * page)
        c = min(max(int(count[b]), 0), tokens, n)
        if c == 0:
            continue
        pid = table[b, :(n + page - 1) // page].long()
        good = ((pid >= 0) & (pid < pages)).repeat_interleave(page)[:n]
        pid = pid.clamp(0, pages - 1)
        pid = torch.where((table[b, :pid.numel()] >= 0) & (table[b, :pid.numel()] < pages), pid, 0)
        pos = torch.arange(n - c, n)[:, None]
        j = torch.arange(n)[None, :]
        seen = (j <= pos) & good[None, :]
        if window:
            seen &= j > pos - window
        for h in range(heads):
            k, v = kv[pid, h].reshape(-1, dim)[:n], vv[pid, h].reshape(-1, dim)[:n]
            any_seen = seen.any(0)
            k, v = torch.where(any_seen[:, None], k, 0.0), torch.where(any_seen[:, None], v, 0.0)
            for g in range(group):
                x = q[b, :c, h * group + g].double()
                s = torch.where(seen, scale * (x @ k.T), -math.inf)
                some = seen.any(1, keepdim=True)
                top = torch.where(some, s.amax(1, keepdim=True), 0.0)
                p = torch.exp(s - top)
                total = p.sum(1, keepdim=True).clamp(min=1e-300)
                o[b, :c, h * group + g] = torch.where(some, p @ v / total, 0.0)
                # Weights off by 2^-11 (16 bits) and by the scores' own errors, twice (sum and weights); a weight is
                # cut at 2^-25 of the largest scaled one, times a page's largest value, for each key.
                ds = ((dim + 4) * 2.0 ** -23 * scale * (x.abs() @ k.abs().T) + s.abs().nan_to_num(posinf=0) * 2.0 ** -22).nan_to_num()
                rel = 2.0 ** -11 + 2 * (ds * seen).amax(1, keepdim=True) + 2.0 ** -18
                cut = n * 2.0 ** -25 * 2 * float(v.abs().max()) * 2
                off[b, :c, h * group + g] = torch.where(some, rel * (p @ v.abs()) / total + cut / total, 0.0)
    return o, off


def attention_case(ops, dim, page, heads, group, tokens, lengths, window=0, dtype=BF16, count=None, seed=0, holes=False):
    batch, longest = len(lengths), max(max(lengths), 1)
    columns = (longest + page - 1) // page + 1
    pages = batch * columns + 3
    cache = filled_cache(ops, pages, heads, page, dim, seed)
    gen = torch.Generator().manual_seed(seed + 1)
    table = torch.randperm(pages, generator=gen)[:batch * columns].reshape(batch, columns).to(torch.int32)
    if holes:
        table[:, 1::3] = -1
        table[0, 0] = pages + 5
    length = torch.tensor(lengths, dtype=torch.int32)
    n = torch.full((batch,), tokens, dtype=torch.int32) if count is None else torch.tensor(count, dtype=torch.int32)
    q = normal(seed + 2, batch, tokens, heads * group, dim).to(dtype)
    o = ops.attention_fp8(q.to(DEV), *cache, table.to(DEV), length.to(DEV), None if count is None else n.to(DEV), window=window)
    want, off = attention_reference(q, cache, table, length, n, window, 1 / math.sqrt(dim))
    near(o, want, off)
    return o


@pytest.mark.parametrize("dim", [16, 48, 64, 80, 128, 144, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attention_one_token(ops, dim, page, dtype):
    attention_case(ops, dim, page, 2, 4, 1, [0, 1, 15, 16, 17, 63, 64, 65, 130, 700], dtype=dtype, seed=dim)


@pytest.mark.parametrize("heads,group", [(1, 1), (1, 7), (2, 8), (1, 16), (1, 17), (3, 5), (1, 40)])
@pytest.mark.parametrize("tokens", [1, 2, 9])
def test_attention_heads_and_tokens(ops, heads, group, tokens):
    attention_case(ops, 64, 32, heads, group, tokens, [tokens, 100, 333], seed=heads * group)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("tokens,lengths", [(130, [130, 300, 131]), (65, [65, 64, 800]), (257, [257])])
def test_attention_many_tokens(ops, dim, tokens, lengths):
    attention_case(ops, dim, 64, 1, 2, tokens, lengths, count=[min(tokens, n) for n in lengths], seed=tokens)


@pytest.mark.parametrize("window", [1, 16, 63, 64, 100])
@pytest.mark.parametrize("tokens", [1, 40])
def test_attention_window(ops, window, tokens):
    attention_case(ops, 64, 16, 2, 2, tokens, [tokens, 90, 500], window=window, seed=window)


def test_attention_ragged_counts_and_empty_rows(ops):
    o = attention_case(ops, 64, 32, 2, 3, 6, [0, 3, 200, 6, 50], count=[0, 3, 1, 0, 6], seed=5)
    assert torch.all(o[0] == 0) and torch.all(o[1, 3:] == 0) and torch.all(o[2, 1:] == 0) and torch.all(o[3] == 0)


@pytest.mark.parametrize("tokens", [1, 20])
def test_attention_pages_outside_the_cache_are_not_seen(ops, tokens):
    attention_case(ops, 64, 32, 1, 4, tokens, [20, 100, 400], holes=True, seed=8)


@pytest.mark.parametrize("lengths", [[20000], [9000, 17, 12345]])
def test_attention_long_axis(ops, lengths):
    """Long enough that the keys are split and joined."""
    attention_case(ops, 128, 64, 1, 4, 1, lengths, seed=3)


def test_attention_weights_far_below_the_largest(ops):
    """One key with a large weight, very many with small ones that add up to as much."""
    dim, page, n = 64, 128, 8192
    cache = ops.kv_cache(n // page, 1, page, dim, DEV)
    k, v = torch.zeros(1, n, 1, dim), torch.full((1, n, 1, dim), -1.0)
    k[0, 100, 0, 0] = 8 * 13 * math.log(2)                          # weight 2^13 times the others'
    v[0, 100] = 1.0
    table = torch.arange(n // page, dtype=torch.int32)[None]
    ops.kv_cache_append(k.to(DEV), v.to(DEV), *cache, table.to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    q = torch.zeros(1, 1, 1, dim, dtype=F16)
    q[..., 0] = 1
    length = torch.tensor([n], dtype=torch.int32)
    o = ops.attention_fp8(q.to(DEV), *cache, table.to(DEV), length.to(DEV))
    want, off = attention_reference(q, cache, table, length, torch.ones(1), 0, 1 / 8)
    near(o, want, off)


def test_attention_scales_of_pages_far_apart(ops):
    """Pages whose value scales are 2^+-40 apart: what the last sees decides alone, and the sums stay finite."""
    dim, page = 64, 16
    cache = filled_cache(ops, 6, 1, page, dim)
    for i, e in enumerate((87, 127, 167, 127, 90, 160)):
        cache[3].view(torch.uint8)[i] = e
    table = torch.arange(6, dtype=torch.int32)[None]
    q = normal(1, 1, 90, 2, dim).to(BF16)
    length = torch.tensor([90], dtype=torch.int32)
    o = ops.attention_fp8(q.to(DEV), *cache, table.to(DEV), length.to(DEV))
    # Row by row, since a row's largest value sets what is cut.
    for t in (0, 10, 15, 16, 40, 89):
        n = torch.tensor([t + 1], dtype=torch.int32)
        want, off = attention_reference(q[:, t:t + 1], cache, table, n, torch.ones(1), 0, 1 / 8)
        near(o[:, t:t + 1], want, off)


def test_attention_ignores_what_pages_hold_past_the_end(ops):
    """NaN bytes past a sequence's last token, and in keys and values that a window hides from every query."""
    dim, page = 64, 32
    cache = filled_cache(ops, 8, 2, page, dim)
    table = torch.arange(8, dtype=torch.int32).reshape(2, 4)
    length = torch.tensor([37, 90], dtype=torch.int32)
    q = normal(2, 2, 1, 4, dim).to(BF16)
    args = (table.to(DEV), length.to(DEV))
    whole, windowed = ops.attention_fp8(q.to(DEV), *cache, *args), ops.attention_fp8(q.to(DEV), *cache, *args, window=20)
    k8, v8 = cache[0].view(torch.uint8), cache[1].view(torch.uint8)
    for b, n in enumerate((37, 90)):
        for slot in range(n, 128):
            k8[b * 4 + slot // page, :, slot % page] = 0x7F
            v8[b * 4 + slot // page, :, :, slot % page] = 0xFF
    got = ops.attention_fp8(q.to(DEV), *cache, *args)
    assert same(got, whole)
    for b, n in enumerate((37, 90)):
        for slot in range(0, n - 20):
            k8[b * 4 + slot // page, :, slot % page] = 0x7F
            v8[b * 4 + slot // page, :, :, slot % page] = 0xFF
    got = ops.attention_fp8(q.to(DEV), *cache, *args, window=20)
    assert same(got, windowed)


def test_attention_infinite_and_nan_queries(ops):
    dim = 64
    cache = filled_cache(ops, 4, 1, 32, dim)
    table, length = torch.arange(4, dtype=torch.int32)[None].to(DEV), torch.tensor([100], dtype=torch.int32, device=DEV)
    q = normal(2, 1, 1, 4, dim).to(BF16)
    want = ops.attention_fp8(q.to(DEV), *cache, table, length)
    q[0, 0, 2, 5] = float("nan")
    got = ops.attention_fp8(q.to(DEV), *cache, table, length)
    assert torch.isnan(got[0, 0, 2]).all()
    for h in (0, 1, 3):
        assert torch.equal(got[0, 0, h], want[0, 0, h])


def test_attention_strides(ops):
    dim, heads, group, tokens = 80, 2, 3, 5
    cache = filled_cache(ops, 8, heads, 32, dim)
    table = torch.arange(8, dtype=torch.int32).reshape(2, 4)
    wide = torch.full((2, 9), -1, dtype=torch.int32)
    wide[:, 2:6] = table
    length = torch.tensor([128, 77], dtype=torch.int32, device=DEV)
    q = normal(2, tokens, 2, heads * group, dim + 7).to(F16).to(DEV)
    view = q.transpose(0, 1)[..., 3:3 + dim]
    got = ops.attention_fp8(view, *cache, wide.to(DEV)[:, 2:6], length)
    assert torch.equal(got, ops.attention_fp8(view.contiguous(), *cache, table.to(DEV), length))


def test_attention_over_a_cache_past_4_gib(ops):
    """Page offsets beyond 2^32 bytes, in keys and values."""
    heads, page, dim = 8, 128, 128
    pages = (2 ** 32 + 2 ** 28) // (heads * page * dim)
    cache = ops.kv_cache(pages, heads, page, dim, DEV)
    last = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device=DEV)
    k, v = (normal(i, 1, 300, heads, dim).to(DEV) for i in (1, 2))
    ops.kv_cache_append(k, v, *cache, last, torch.zeros(1, dtype=torch.int32, device=DEV))
    small = ops.kv_cache(3, heads, page, dim, DEV)
    table, length = torch.arange(3, dtype=torch.int32, device=DEV)[None], torch.tensor([300], dtype=torch.int32, device=DEV)
    ops.kv_cache_append(k, v, *small, table, torch.zeros(1, dtype=torch.int32, device=DEV))
    q = normal(3, 1, 1, heads, dim).to(BF16).to(DEV)
    assert torch.equal(ops.attention_fp8(q, *cache, last, length), ops.attention_fp8(q, *small, table, length))


# ---------------------------------------------------------------------------
# Streams, graphs, refusals.

def test_other_streams_and_graphs(ops):
    """On a stream of the caller's, and replayed from a graph, between the caller's own work: the eager results."""
    x, w = normal(1, 8, 512).to(BF16).to(DEV), torch.ones(512, dtype=BF16, device=DEV)
    w8, ws = ops.quantize_weights_fp8(normal(2, 256, 512).to(DEV))
    cache = filled_cache(ops, 64, 1, 32, 64)
    table, length = torch.arange(64, dtype=torch.int32, device=DEV)[None].repeat(8, 1), torch.full((8,), 1900, dtype=torch.int32, device=DEV)

    def step():
        y, s, _, _ = ops.rms_norm(x, w)
        q = ops.linear_fp8(y, s, w8, ws).view(8, 1, 4, 64)
        ops.kv_cache_append(q[:1, :, :1], q[:1, :, 1:2], *cache, table[:1], length[:1])
        return ops.attention_fp8(q, *cache, table, length)

    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step()
    s.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        x.copy_(normal(10 + i, 8, 512).to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step())


def test_refusals(ops):
    x = torch.zeros(4, 256, dtype=BF16, device=DEV)
    w = torch.ones(256, dtype=BF16, device=DEV)
    x8, xs = ops.quantize_fp8(x)
    w8, ws = ops.quantize_weights_fp8(x)
    cache = ops.kv_cache(4, 2, 16, 64, DEV)
    table, one = torch.zeros(1, 4, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    q = torch.zeros(1, 1, 4, 64, dtype=BF16, device=DEV)
    k = torch.zeros(1, 1, 2, 64, dtype=BF16, device=DEV)
    bad = [
        lambda: ops.rms_norm(x.cpu(), w),
        lambda: ops.rms_norm(x.int(), w),
        lambda: ops.rms_norm(x, w[:5]),
        lambda: ops.rms_norm(x, w.to(F16)),
        lambda: ops.rms_norm(x, w, x[:2]),
        lambda: ops.rms_norm(x.t(), w[:4]),
        lambda: ops.rms_norm(x, w, eps=-1.0),
        lambda: ops.rms_norm(x, w, eps=float("nan")),
        lambda: ops.rms_norm(torch.zeros(1, 70000, device=DEV), torch.ones(70000, device=DEV)),
        lambda: ops.rms_norm_backward(x, x.to(F16), w, torch.ones(4, device=DEV)),
        lambda: ops.rms_norm_backward(x, x, w, torch.ones(3, device=DEV)),
        lambda: ops.quantize_fp8(x, x[:, :8]),
        lambda: ops.quantize_fp8(x8),
        lambda: ops.shift_weights_to_fp8(torch.zeros(4, 3, dtype=torch.int32, device=DEV), 100),
        lambda: ops.linear_fp8(x8, xs, w8[:, :128], ws[:, :1]),
        lambda: ops.linear_fp8(x8, xs[:, :1], w8, ws),
        lambda: ops.linear_fp8(x8, xs, w8, ws, out_dtype=torch.int32),
        lambda: ops.linear_fp8(x8, xs, w8, ws, torch.zeros(3, device=DEV)),
        lambda: ops.linear_fp8(x, xs, w8, ws),
        lambda: ops.linear_fp8_backward_data(x8, xs, w8, ws),
        lambda: ops.kv_cache(4, 2, 24, 64),
        lambda: ops.kv_cache_append(k, k, *cache, table, None),
        lambda: ops.kv_cache_append(k, k[..., :32], *cache, table, one),
        lambda: ops.kv_cache_append(k, k, *cache, table.long(), one),
        lambda: ops.attention_fp8(q.float(), *cache, table, one),
        lambda: ops.attention_fp8(q[:, :, :3], *cache, table, one),
        lambda: ops.attention_fp8(q[..., :32], *cache, table, one),
        lambda: ops.attention_fp8(q, *cache, table, one.cpu()),
        lambda: ops.attention_fp8(q, *cache, table, one, window=-1),
        lambda: ops.attention_fp8(q, *cache, table, one, scale=float("inf")),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((TypeError, ValueError, ops.DeepShiftError)):
            f()
            pytest.fail(f"case {i} was accepted")
