"""The 8-bit decoder operators on the GPU at the ends of their ranges: last tiles of one
row, sequences beyond their table, weights far below the largest, values that are no
numbers. Definitions in 64 bits and tolerances as in test_gpu_fp8.
"""
import math

import numpy as np  # noqa: F401
import pytest
import torch

from .test_gpu_decoder import build as build_decoder
from .test_gpu_fp8 import BF16, DEV, E4M3, E5M2, F16, F32, filled_cache, near, normal, operands, product_terms, value  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_1905_13298_amd import ops as o
    return o


# ---------------------------------------------------------------------------
# Product.

@pytest.mark.parametrize("m,n", [(65, 65), (1025, 2049), (2177, 2049), (3841, 3841)])
@pytest.mark.parametrize("k", [1, 16, 100, 128, 272])
def test_product_tiles_of_one_row(ops, m, n, k):
    """Last tiles of one row of x and of w (tiles of 64, of 128 in four and in two stages, of 256), with
    fewer steps than a tile sends for ahead: their buffers are a row, shorter than those steps' offsets."""
    x8, xs, w8, ws = operands(ops, m, n, k, E4M3, k)
    y = ops.linear_fp8(x8, xs, w8, ws).cpu()
    rows = torch.tensor([0, 1, m // 2, m - 2, m - 1])
    x, w = value(x8, xs)[rows], value(w8, ws, 128)
    near(y[rows], x @ w.T, product_terms(x, w, k, False))


@pytest.mark.parametrize("m", [5, 70, 1100])
@pytest.mark.parametrize("out", [BF16, F16, F32])
def test_product_nan_scales(ops, m, out):
    """A scale of NaN makes its block's products NaN: one row (x) or 128 columns (w) of y, in every output type."""
    n, k = 400, 700
    x8, xs, w8, ws = operands(ops, m, n, k, E4M3)
    want = ops.linear_fp8(x8, xs, w8, ws, out_dtype=out)
    xs.view(torch.uint8)[m // 2, 3] = 255
    ws.view(torch.uint8)[1, 5] = 255
    got = ops.linear_fp8(x8, xs, w8, ws, out_dtype=out)
    nan = torch.zeros(m, n, dtype=torch.bool, device=DEV)
    nan[m // 2], nan[:, 128:256] = True, True
    assert torch.equal(got.isnan(), nan) and torch.equal(got[~nan], want[~nan])


# ---------------------------------------------------------------------------
# Attention.

def definition(q, cache, table, length, count, window, scale):
    """(o, what it may be off by) of the definition in 64 bits: query i < count of a sequence is at position
    length - count + i and sees the keys up to there, the last `window` of them, that the table has a page for."""
    k8, v8, ks, vs = (t.cpu() for t in cache)
    pages, heads, page, dim = k8.shape
    batch, tokens, hq, _ = q.shape
    o, off = torch.zeros(batch, tokens, hq, dim, dtype=torch.float64), torch.zeros(batch, tokens, hq, dim, dtype=torch.float64)
    for b in range(batch):
        c, n = min(max(int(count[b]), 0), tokens), min(max(int(length[b]), 0), table.shape[1] * page)
        if c == 0 or n == 0:
            continue
        pid = table[b, :(n + page - 1) // page].long()
        good = ((pid >= 0) & (pid < pages)).repeat_interleave(page)[:n]
        pid = torch.where((pid >= 0) & (pid < pages), pid, 0)
        pos = (max(int(length[b]), 0) - c + torch.arange(c))[:, None]
        j = torch.arange(n)[None, :]
        seen = (j <= pos) & good[None, :]
        if window:
            seen &= j > pos - window
        some = seen.any(1, keepdim=True)
        for h in range(heads):
            key = torch.exp2(ks.view(torch.uint8)[pid, h].double() - 127).repeat_interleave(page)[:n]
            val = torch.exp2(vs.view(torch.uint8)[pid, h].double() - 127).repeat_interleave(page)[:n]
            k = torch.where(seen.any(0)[:, None], k8[pid, h].double().reshape(-1, dim)[:n] * key[:, None], 0.0)
            v = torch.where(seen.any(0)[:, None], v8[pid, h].double().transpose(1, 2).reshape(-1, dim)[:n], 0.0)     # without the scale
            nan = v.isnan()
            v = v.nan_to_num(0.0)
            for g in range(hq // heads):
                x = q[b, :c, h * (hq // heads) + g].double()
                s = torch.where(seen, scale * (x @ k.T), -math.inf)
                p = torch.exp(s - torch.where(some, s.amax(1, keepdim=True), 0.0))
                total = p.sum(1, keepdim=True).clamp(min=1e-300)
                p = p * val
                out = torch.where(some, p @ v / total, 0.0)
                o[b, :c, h * (hq // heads) + g] = torch.where(seen.double() @ nan.double() > 0, math.nan, out)
                # Scores in 32 bits; weights rounded to 2^-11 each for itself (their errors add up as squares do: 6
                # deviations of a uniform error); below 2^-23 of the largest one, to 2^-34 of it.
                ds = ((dim + 4) * 2.0 ** -23 * scale * (x.abs() @ k.abs().T) + s.abs().nan_to_num(posinf=0) * 2.0 ** -22).nan_to_num()
                rel = 2 * (ds * seen).amax(1, keepdim=True) + 2.0 ** -20
                squares = 6 / math.sqrt(3) * (torch.maximum(p * 2.0 ** -11, p.amax(1, keepdim=True) * 2.0 ** -34 * seen).square() @ v.square()).sqrt()
                off[b, :c, h * (hq // heads) + g] = torch.where(some, (rel * (p @ v.abs()) + squares) / total, 0.0)
    return o, off


def agree(o, want, off):
    nan = want.isnan()
    assert torch.equal(o.cpu().isnan(), nan)
    near(o.cpu().nan_to_num(0.0), want.nan_to_num(0.0), off)


def pages_of(ops, batch, columns, heads, page, dim, seed=0):
    cache = filled_cache(ops, batch * columns + 2, heads, page, dim, seed)
    table = torch.randperm(batch * columns + 2, generator=torch.Generator().manual_seed(seed))[:batch * columns].reshape(batch, columns)
    return cache, table.to(torch.int32)


def attend(ops, q, cache, table, length, count=None, window=0):
    length = torch.tensor(length, dtype=torch.int32)
    c = torch.tensor([q.shape[1]] * len(length) if count is None else count, dtype=torch.int32)
    o = ops.attention_fp8(q.to(DEV), *cache, table.to(DEV), length.to(DEV), None if count is None else c.to(DEV), window=window)
    return o, *definition(q, cache, table, length, c, window, 1 / math.sqrt(q.shape[3]))


@pytest.mark.parametrize("tokens,group", [(1, 2), (5, 2), (10, 4), (150, 2)])
@pytest.mark.parametrize("window", [0, 7, 40])
def test_attention_of_sequences_past_their_table(ops, tokens, group, window):
    """Queries keep their positions where their own keys found no room, where counts are over the tokens or the length, and
    where lengths are negative."""
    columns, page, dim = 4, 16, 64
    cap = columns * page
    length = [cap + tokens - 1, cap + 1, cap + 6, cap, 3, 0, -9, cap + 500, 30]
    count = [tokens, tokens, tokens, tokens + 3, 5, tokens, 1, tokens, -2]
    cache, table = pages_of(ops, len(length), columns, 2, page, dim)
    q = normal(3, len(length), tokens, 2 * group, dim).to(BF16)
    agree(*attend(ops, q, cache, table, length, count, window))

def shared_pages(ops, k, v, page, batch):
    """A cache of one sequence [n, dim] that `batch` sequences share, enough that no sequence is split."""
    n, dim = k.shape
    cache = ops.kv_cache((n + page - 1) // page, 1, page, dim, DEV)
    table = torch.arange(cache[0].shape[0], dtype=torch.int32)[None]
    ops.kv_cache_append(k[None, :, None].to(DEV), v[None, :, None].to(DEV), *cache, table.to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    return cache, table.repeat(batch, 1)


def one_of_many(ops, q, cache, table, n, window=0):
    """The first of many equal sequences, against the definition."""
    batch = table.shape[0]
    length = torch.full((batch,), n, dtype=torch.int32)
    o = ops.attention_fp8(q.to(DEV).expand(batch, *q.shape[1:]), *cache, table.to(DEV), length.to(DEV), window=window)
    assert bool((o == o[:1]).all())
    agree(o[:1], *definition(q, cache, table[:1], length[:1], torch.tensor([q.shape[1]]), window, 1 / math.sqrt(q.shape[3])))


@pytest.mark.parametrize("low,high", [(-18, -20), (-20, -24), (-23, -27)])
@pytest.mark.parametrize("tokens,group", [(1, 4), (8, 4), (40, 4)])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_of_a_sink_and_many_small_weights(ops, low, high, tokens, group, dim):
    """A dominant key without a value; all that comes out is of keys with 2^low .. 2^high of its weight."""
    n = 16384
    k = torch.zeros(n, dim)
    k[:, 0] = (torch.rand(n, generator=torch.Generator().manual_seed(1)) * (high - low) + low) * math.log(2) + 8
    k[:, 1] = normal(2, n)
    k[0, 0], k[0, 1] = 8, 0
    v = normal(3, n, dim) * 1024
    v[0] = 0
    cache, table = shared_pages(ops, k, v, 64, 512)
    q = torch.zeros(1, tokens, group, dim, dtype=F16)
    q[..., 0], q[..., 1] = math.sqrt(dim), 0.25
    one_of_many(ops, q, cache, table, n)


@pytest.mark.parametrize("times", [12, 16])
@pytest.mark.parametrize("tokens,group", [(1, 4), (8, 4), (40, 4)])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_beside_a_large_value_that_no_query_sees(ops, times, tokens, group, dim):
    """A value before the window that is 2^times as large as the others sets its page's scale."""
    n, page = 8192, 64
    window = n - tokens - 30
    k, v = normal(4, n, dim), normal(5, n, dim) * 16
    v[3] *= 2.0 ** times
    cache, table = shared_pages(ops, k, v, page, 512)
    q = (normal(6, 1, tokens, group, dim)).to(F16)
    one_of_many(ops, q, cache, table, n, window)


@pytest.mark.parametrize("dim,tokens,group,page,length", [(64, 1, 4, 16, 40), (256, 1, 3, 64, 300), (64, 5, 2, 16, 40), (128, 3, 5, 64, 300), (256, 2, 1, 32, 33), (64, 70, 2, 16, 90), (128, 200, 3, 64, 700),
                                                          (256, 40, 1, 128, 250), (80, 33, 2, 32, 33), (128, 9, 1, 64, 9000), (128, 30, 2, 64, 9000)])
@pytest.mark.parametrize("window", [0, 20])
def test_attention_nan_values_reach_the_queries_that_see_them(ops, dim, tokens, group, page, length, window):
    heads, columns = 2, (length + page - 1) // page
    cache, table = pages_of(ops, 2, columns, heads, page, dim, seed=7)
    lengths, counts = [length, length - 3], [tokens, tokens - 1]
    v8 = cache[1].view(torch.uint8)
    for b, n in enumerate(lengths):
        # In the last tokens, in the first ones that a window hides from some, and one before all of those.
        for i, t in enumerate(sorted({max(n - tokens - 30, 0), max(n - tokens - 12, 0), n - tokens, n - tokens // 2 - 1, n - 1})):
            v8[int(table[b, t // page]), i % heads, (5 * i + 3) % dim, t % page] = 0x7F if i % 2 else 0xFF
    q = normal(8, 2, tokens, heads * group, dim).to(BF16)
    o, want, off = attend(ops, q, cache, table, lengths, counts, window)
    agree(o, want, off)
    assert bool(want.isnan().any()) and not bool(want.isnan().all())
    v8.copy_(torch.where((v8 & 0x7F) == 0x7F, torch.zeros_like(v8), v8))
    clean, _, _ = attend(ops, q, cache, table, lengths, counts, window)
    nan = o.isnan()
    assert torch.equal(o[~nan], clean[~nan])


# ---------------------------------------------------------------------------
# Decoder.

def test_decoder_past_its_capacity():
    """A ragged prompt that crosses the capacity: the tokens that found room come out as from a decoder with more of it."""
    make, ps, norm, rng = build_decoder(5, 2, 256, 8, 2, 32, 512, BF16, 3, 64, 16, 0)
    room, ps, norm, rng = build_decoder(5, 2, 256, 8, 2, 32, 512, BF16, 3, 96, 16, 0)
    small, large = make(), room()
    assert (small.capacity, large.capacity) == (64, 96)
    x = torch.from_numpy(rng.standard_normal((3, 80, 256))).to(DEV, BF16)
    first = torch.tensor([60, 10, 33], dtype=torch.int32, device=DEV)
    assert torch.equal(small(x[:, :60], first), large(x[:, :60], first))
    got, want = small(x[:, 60:72]), large(x[:, 60:72])
    for b, n in enumerate((4, 12, 12)):
        assert torch.equal(got[b, :n], want[b, :n])
    assert small.length.tolist() == large.length.tolist() == [72, 22, 45]
    # A count above the tokens means all of them.
    many = torch.full((3,), 9, dtype=torch.int32, device=DEV)
    got, want = small(x[:, 72:74], many), large(x[:, 72:74])
    assert torch.equal(got[1:], want[1:]) and small.length.tolist() == [74, 24, 47]


def test_decoder_is_unchanged_by_a_refused_call():
    make, ps, norm, rng = build_decoder(6, 1, 256, 8, 2, 32, 512, BF16, 2, 64, 16, 0)
    model, other = make(), make()
    x = torch.from_numpy(rng.standard_normal((2, 4, 256))).to(DEV, BF16)
    two = torch.full((2,), 2, dtype=torch.int32, device=DEV)
    bad = [lambda: model(x.float()), lambda: model(x.half()), lambda: model(x.cpu()), lambda: model(x[:1]), lambda: model(x[0]), lambda: model(x[..., :128]),
           lambda: model(x, two.long()), lambda: model(x, two[:1]), lambda: model(x, two.cpu()), lambda: model(x, two[:, None]), lambda: model(x, 2)]
    for i, call in enumerate(bad):
        with pytest.raises((TypeError, ValueError)):
            call()
            pytest.fail(f"case {i} was accepted")
        assert model.length.tolist() == [0, 0], i
    for a, b in zip(model.caches[0], other.caches[0]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(model(x, two), other(x, two)) and model.length.tolist() == [2, 2]


def test_decoder_without_tokens():
    """No tokens: no rows come out and nothing changes."""
    make, ps, norm, rng = build_decoder(6, 2, 256, 8, 2, 32, 512, BF16, 2, 64, 16, 0)
    model = make()
    x = torch.from_numpy(rng.standard_normal((2, 4, 256))).to(DEV, BF16)
    want = make()(x)
    assert model(x[:, :0]).shape == (2, 0, 256) and model.length.tolist() == [0, 0]
    none = model(x, torch.zeros(2, dtype=torch.int32, device=DEV))
    assert none.shape == x.shape and model.length.tolist() == [0, 0]
    assert torch.equal(model(x), want)


# ---------------------------------------------------------------------------
# Weights.

@pytest.mark.parametrize("rows,cols,bits", [(65536, 5, 5), (131100, 20, 4)])
def test_shift_weights_of_many_rows(ops, rows, cols, bits):
    rng = np.random.default_rng(rows)
    codes = (rng.integers(0, 2 ** (bits - 1) - 1, (rows, cols)) + 16 * rng.integers(0, 2, (rows, cols))).astype(np.uint8)
    w8, s = ops.shift_weights_to_fp8(torch.from_numpy(ops.pack_shift_weights(codes, bits).view(np.int32)).to(DEV), cols, bits)
    want = np.where(codes & 16, -1.0, 1.0) * 2.0 ** -(codes & 15).astype(float)
    assert np.array_equal(w8.cpu().double().numpy(), want) and s.shape == ((rows + 127) // 128, 1)
    with pytest.raises(ops.DeepShiftError):
        ops.shift_weights_to_fp8(torch.zeros(0, 2, dtype=torch.int32, device=DEV), 12, 5)


def test_shift_weights_of_one_row_of_2_to_the_31(ops):
    """The last block's columns pass 31 bits: they are written up to a multiple of 8 and no further."""
    cols = 2 ** 31 - 1
    words = ops.packed_row_words(cols, 5)
    wp = torch.full((1, words), 0x01084210, dtype=torch.int32, device=DEV)
    last = torch.randint(0, 2 ** 30, (100,), generator=torch.Generator().manual_seed(1)).int()
    wp[0, -100:] = last.to(DEV)
    buffer = torch.full((2 ** 31 + 8192,), 0xAA, dtype=torch.uint8, device=DEV)
    ops.call("ds_shift_weights_to_fp8", wp.data_ptr(), buffer.data_ptr() + 4096, 1, cols, 2 ** 31, 0, torch.cuda.current_stream().cuda_stream)
    assert torch.all(buffer[:4096] == 0xAA) and torch.all(buffer[4096 + 2 ** 31:] == 0xAA)
    n = cols - (words - 100) * 6
    codes = torch.stack([(last >> (5 * j)) & 31 for j in range(6)], 1).reshape(-1)[:n]
    want = torch.where((codes & 15) == 15, 0.0, torch.where(codes >= 16, -1.0, 1.0) * torch.exp2(-(codes & 15).float()))
    got = buffer[4096 + cols - n:4096 + cols].cpu().view(E5M2).float()
    assert torch.equal(got, want) and int(buffer[4096 + cols]) == 0


# ---------------------------------------------------------------------------
# Norm.

@pytest.mark.parametrize("cols", [1, 300, 1001, 3002])
def test_norm_writes_zeros_behind_a_row_without_numbers(ops, cols):
    x = normal(4, 3, cols).to(BF16)
    x[1, 0] = float("nan")
    x[2] = 0
    y, s, _, _ = ops.rms_norm(x.to(DEV), torch.ones(cols, device=DEV), eps=0.0)
    whole = y.view(torch.uint8).as_strided((3, (cols + 7) // 8 * 8), (y.stride(0), 1)).cpu()
    assert torch.all(whole[:, cols:] == 0)
    assert torch.all(whole[1:, :cols] & 0x7F == 0x7F)
