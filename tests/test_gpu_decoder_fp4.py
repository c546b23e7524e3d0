"""The decoder with rotated heads and a 4-bit cache on the GPU.

Against its operators called one by one the results are equal. Against the same layers in 64 bits without any rounding: an
8-bit rounding (E4M3) is off by at most 2^-4 of an element, four of them a layer (norm, attention's output, norm, gated values). A
cached element's 4-bit step is at most half of it where its block's scale leaves it at 1 or more and 0.5 below; roundings are spread
evenly over a step, 1 / sqrt(12) of it on average: 0.15 of an element, or of the scale, which is less than the root mean square of a
block of normal elements. Twice that square, keys and values alike, with keys' errors moving weights by as much as themselves: sqrt(4
* 2^-8 + 2 * 2 * 0.15^2) = 0.33 of the root mean square of what attention adds, a layer; so for the outputs 0.33 sqrt(layers) at most.
"""
import math

import numpy as np
import pytest
import torch

from .test_gpu_decoder import exact_weights, layer_params, norm64

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64


def rotate64(x, positions, frequencies, sections, interleaved):
    """x [tokens, heads, dim], positions [tokens] or [axes, tokens]."""
    n = frequencies.numel()
    p = positions.double() if positions.dim() == 2 else positions.double()[None]
    axis = torch.tensor([i for i, k in enumerate(sections or (n,)) for _ in range(k)])
    a = (p[axis].T * frequencies.cpu().double())[:, None]
    i = torch.arange(n)
    f, s = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    y = x.clone()
    y[..., f] = x[..., f] * torch.cos(a) - x[..., s] * torch.sin(a)
    y[..., s] = x[..., s] * torch.cos(a) + x[..., f] * torch.sin(a)
    return y


def layer64(x, p, r, positions, heads, kv_heads, dim, inner, window):
    """One sequence [tokens, hidden] -> the layer's output."""
    t, hidden = x.shape
    qkv = (norm64(x, p["norm1"]) @ exact_weights(p["qkv"], hidden).T).view(t, -1, dim)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], dim=1)
    q, k = (rotate64(norm64(a, w) if w is not None else a, positions, r.frequencies, r.sections, r.interleaved) for a, w in ((q, r.q_norm), (k, r.k_norm)))
    k, v = (a.repeat_interleave(heads // kv_heads, 1) for a in (k, v))
    s = (q.transpose(0, 1) @ k.permute(1, 2, 0)) / math.sqrt(dim)
    i = torch.arange(t)
    seen = i[None, :] <= i[:, None]
    if window:
        seen &= i[None, :] > i[:, None] - window
    o = torch.softmax(s.masked_fill(~seen, -math.inf), -1) @ v.transpose(0, 1)
    x = x + o.transpose(0, 1).reshape(t, -1) @ exact_weights(p["out"], heads * dim).T
    gate, up = (norm64(x, p["norm2"]) @ exact_weights(p["gate_up"], hidden).T).chunk(2, 1)
    return x + (gate / (1 + torch.exp(-gate)) * up) @ exact_weights(p["down"], inner).T


def build(seed, layers, hidden, heads, kv_heads, dim, inner, dtype, batch, tokens, page, window, sections=None, interleaved=False, norms=True,
          cache_bits=4):
    from paper_1905_13298_amd import decoder, ops
    rng = np.random.default_rng(seed)
    ps = [layer_params(rng, hidden, heads, kv_heads, dim, inner, dtype) for _ in range(layers)]
    f = ops.rotary_frequencies(dim // 2)
    weight = lambda: torch.from_numpy(1 + 0.2 * rng.standard_normal(dim)).to(DEV, dtype) if norms else None  # noqa: E731
    rs = [decoder.Rotary(f, weight(), weight(), sections, interleaved) for _ in range(layers)]
    norm = torch.from_numpy(1 + 0.2 * rng.standard_normal(hidden)).to(DEV, dtype)
    made = [decoder.DecoderLayer(p, heads, kv_heads, dim, inner, window=window, rotary=r, cache_bits=cache_bits) for p, r in zip(ps, rs)]
    return (lambda: decoder.Decoder(made, norm, batch, tokens, page)), ps, rs, norm, rng


@pytest.mark.parametrize("layers,hidden,heads,kv_heads,dim,inner,dtype,page,window,sections,interleaved,cache_bits", [
    (1, 256, 8, 2, 32, 512, BF16, 16, 0, None, False, 4), (2, 200, 5, 5, 48, 330, F16, 32, 0, (8, 8, 8), True, 4),
    (2, 512, 8, 1, 128, 1024, BF16, 64, 24, None, False, 4), (1, 256, 4, 2, 80, 256, BF16, 16, 0, None, False, 8),
])
def test_decoder(layers, hidden, heads, kv_heads, dim, inner, dtype, page, window, sections, interleaved, cache_bits):
    batch, prompt, single = 3, 70, 5
    make, ps, rs, norm, rng = build(1, layers, hidden, heads, kv_heads, dim, inner, dtype, batch, prompt + single, page, window, sections, interleaved,
                                    cache_bits=cache_bits)
    x = torch.from_numpy(rng.standard_normal((batch, prompt + single, hidden))).to(dtype)
    counts = torch.tensor([prompt, 1, 33])
    at = None
    if sections:
        at = torch.from_numpy(rng.integers(0, 40, (len(sections), batch, prompt + single))).to(torch.int32)
    part = lambda lo, hi: None if at is None else at[:, :, lo:hi].to(DEV)  # noqa: E731
    model = make()
    first = model(x[:, :prompt].to(DEV), counts.int().to(DEV), positions=part(0, prompt))
    steps = [model(x[:, prompt + i:prompt + i + 1].to(DEV), positions=part(prompt + i, prompt + i + 1)) for i in range(single)]
    assert model.length.tolist() == (counts + single).tolist()
    bound = 0.33 * math.sqrt(layers)
    for b in range(batch):
        n = int(counts[b])
        y = torch.cat([x[b, :n], x[b, prompt:]]).double()
        where = torch.arange(n + single) if at is None else torch.cat([at[:, b, :n], at[:, b, prompt:]], 1)
        for p, r in zip(ps, rs):
            y = layer64(y, p, r, where, heads, kv_heads, dim, inner, window)
        y = norm64(y, norm)
        got = torch.cat([first[b, :n]] + [s[b] for s in steps]).cpu().double()
        for which in (slice(0, n), slice(n, n + single)):
            err = (got[which] - y[which]).square().mean().sqrt() / y[which].square().mean().sqrt()
            assert err <= bound, (b, which, float(err), bound)


def test_a_layer_is_its_operators_one_by_one():
    from paper_1905_13298_amd import ops
    heads, kv, dim, batch = 6, 2, 64, 2
    make, ps, rs, norm, rng = build(5, 1, 256, heads, kv, dim, 512, BF16, batch, 100, 32, 0)
    model, twin = make(), make()
    layer, r = twin.layers[0], rs[0]
    cache = twin.caches[0]
    length = torch.zeros(batch, dtype=torch.int32, device=DEV)
    for tokens in (37, 1, 1, 4):
        x = torch.from_numpy(rng.standard_normal((batch, tokens, 256))).to(DEV, BF16)
        got = model(x)
        qkv, h, _ = layer.qkv(x.reshape(-1, 256))
        q, k, v = qkv.view(batch, tokens, -1, dim).split([heads, kv, kv], dim=2)
        positions = (length[:, None] + torch.arange(tokens, device=DEV)).to(torch.int32)
        q, k = ops.rotary_norm(q, k, positions, r.frequencies, r.q_norm, r.k_norm)
        ops.kv_cache_fp4_append(k, v, *cache, twin.table, length)
        kr, vr = ops.kv_cache_fp4_read(*cache, twin.table, length, tokens)
        assert torch.isfinite(kr).all() and (kr.float() - k.float()).abs().max() <= k.abs().max().float() / 3       # a step is a third of 6
        length = length + tokens
        o = ops.attention_fp4(q, *cache, twin.table, length)
        a = ops.linear_fp8(*ops.quantize_fp8(o.view(batch * tokens, -1)), *layer.out, out_dtype=BF16)
        gu, h, _ = layer.gate_up(a, h)
        gate, up = gu.chunk(2, dim=1)
        y = ops.linear_fp8(*ops.quantize_fp8(up, gate), *layer.down, out_dtype=BF16)
        y, _, _, _ = ops.rms_norm(y, norm, h, quantize=False)
        assert torch.equal(got, y.view(got.shape))
        for mine, theirs in zip(model.caches[0], cache):
            assert torch.equal(mine.view(torch.uint8), theirs.view(torch.uint8))


def test_decoder_graph_and_reset():
    make, _, _, _, rng = build(2, 2, 256, 8, 2, 64, 512, BF16, 2, 64, 16, 0)
    xs = torch.from_numpy(rng.standard_normal((8, 2, 1, 256))).to(DEV, BF16)
    model = make()
    want = [model(x).clone() for x in xs]
    model.reset()
    again = [model(x).clone() for x in xs]
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    model.reset()
    static = xs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = model(static)
    assert model.length.tolist() == [0, 0]
    for x, w in zip(xs, want):
        static.copy_(x)
        graph.replay()
        assert torch.equal(y, w)
        (torch.ones(1000, device=DEV) * 2).sum().item()


@pytest.mark.parametrize("batch,tokens,hidden,heads,kv,dim,dtype", [(1, 9, 256, 4, 2, 64, BF16), (3, 40, 200, 6, 3, 48, F16)])
def test_norm_product_rotation_backward(batch, tokens, hidden, heads, kv, dim, dtype):
    """The way of a training step from the layer's input to its turned queries and keys, and back. Tolerance: dy's 8-bit rounding, 2^-4."""
    make, ps, rs, _, rng = build(3, 1, hidden, heads, kv, dim, 128, dtype, batch, tokens, 16, 0)
    layer, r, p = make().layers[0], rs[0], ps[0]
    draw = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(DEV, dtype)  # noqa: E731
    x, dq, dk, dv = draw(batch * tokens, hidden), draw(batch, tokens, heads, dim), draw(batch, tokens, kv, dim), draw(batch, tokens, kv, dim)
    positions = (torch.arange(tokens, device=DEV)[None] + torch.arange(batch, device=DEV)[:, None] * 100).to(torch.int32)
    qkv, h, rstd = layer.qkv(x)
    q, k, _ = qkv.view(batch, tokens, -1, dim).split([heads, kv, kv], dim=2)
    r(q, k, positions)
    gq, gk, gqn, gkn = r.backward(dq, dk, q, k, positions)
    dx, dn = layer.qkv.backward(torch.cat([gq, gk, dv], 2).view(batch * tokens, -1), h, rstd)
    x64, n64, a64, b64 = (t.cpu().double().requires_grad_() for t in (x, p["norm1"], r.q_norm, r.k_norm))
    y = (x64 / torch.sqrt((x64 * x64).mean(-1, keepdim=True) + 1e-6) * n64 @ exact_weights(p["qkv"], hidden).T).view(batch, tokens, -1, dim)
    loss = (y[:, :, heads + kv:] * dv.cpu().double()).sum()
    for part, w, d in ((y[:, :, :heads], a64, dq), (y[:, :, heads:heads + kv], b64, dk)):
        u = part / torch.sqrt((part * part).mean(-1, keepdim=True) + 1e-6) * w
        loss = loss + sum((rotate64(u[b], positions[b].cpu(), r.frequencies, None, False) * d[b].cpu().double()).sum() for b in range(batch))
    loss.backward()
    for got, want in ((dx, x64.grad), (dn, n64.grad), (gqn, a64.grad), (gkn, b64.grad)):
        err = (got.cpu().double() - want).square().mean().sqrt() / want.square().mean().sqrt()
        assert err <= 2.0 ** -4 * math.sqrt(2), float(err)        # (the forward product's input and dy, both in 8 bits)


def test_a_refused_call_leaves_the_decoder_as_it_was():
    from paper_1905_13298_amd import decoder, ops
    make, ps, rs, norm, rng = build(4, 2, 64, 4, 2, 16, 128, BF16, 2, 40, 16, 0, sections=(4, 4))
    model = make()
    x = torch.zeros(2, 3, 64, dtype=BF16, device=DEV)
    model(x)
    kept = [t.view(torch.uint8).clone() for c in model.caches for t in c]
    at = torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    bad = [at.long(), at[:1], at[None], at[None].expand(3, 2, 3), at.cpu(), at.float()]
    for positions in bad:
        with pytest.raises((TypeError, ValueError)):
            model(x, positions=positions)
    last = model.layers[1]
    rotary = last.rotary
    for worse in (decoder.Rotary(ops.rotary_frequencies(9)), decoder.Rotary(ops.rotary_frequencies(8), torch.ones(15, device=DEV)),
                  decoder.Rotary(ops.rotary_frequencies(8), torch.ones(16, device=DEV, dtype=F16)), decoder.Rotary(ops.rotary_frequencies(8), sections=(4, 5)),
                  decoder.Rotary(ops.rotary_frequencies(8, device="cpu")), decoder.Rotary(ops.rotary_frequencies(8), sections=(2, 2, 2, 1, 1)),
                  decoder.Rotary(ops.rotary_frequencies(8), torch.ones(16, device=DEV), torch.ones(16, device=DEV, dtype=BF16))):
        last.rotary = worse
        with pytest.raises((TypeError, ValueError)):
            model(x)
    last.rotary = rotary
    assert model.length.tolist() == [3, 3]
    assert all(torch.equal(a, b.view(torch.uint8)) for a, b in zip(kept, (t for c in model.caches for t in c)))
    with pytest.raises(ValueError):
        decoder.DecoderLayer(ps[0], 4, 2, 16, 128, cache_bits=5)
    plain = decoder.Decoder([decoder.DecoderLayer(ps[0], 4, 2, 16, 128)], norm, 2, 40, 16)
    with pytest.raises(ValueError):
        plain(x, positions=at)
