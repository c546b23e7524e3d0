"""The decoder of 8-bit operators on the GPU against the same layers in 64 bits without any rounding.

Tolerance: an E4M3 rounding changes an element by at most 2^-4 of itself, independently
of the others, so what a sum of such elements gets is at most 2^-4 of its root mean
square. A layer has five such roundings in a row (norm, cache, attention's output,
norm, gated values; those to 16 bits are 2^-4 of them): 2^-4 sqrt(5 layers) of the
outputs' root mean square. The gradient has one, of dy.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F16 = torch.bfloat16, torch.float16


def shift_codes(rng, rows, cols):
    from paper_1905_13298_amd import ops
    codes = (rng.integers(0, 2, (rows, cols)) << 4 | rng.integers(3, 7, (rows, cols))).astype(np.uint8)
    return torch.from_numpy(ops.pack_shift_weights(codes).view(np.int32)).to(DEV)


def layer_params(rng, hidden, heads, kv_heads, dim, inner, dtype):
    norm = lambda: torch.from_numpy(1 + 0.2 * rng.standard_normal(hidden)).to(DEV, dtype)  # noqa: E731
    return {"norm1": norm(), "norm2": norm(), "qkv": shift_codes(rng, (heads + 2 * kv_heads) * dim, hidden),
            "out": shift_codes(rng, hidden, heads * dim), "gate_up": shift_codes(rng, 2 * inner, hidden),
            "down": shift_codes(rng, hidden, inner)}


def exact_weights(w, cols):
    from paper_1905_13298_amd import ops
    return ops.shift_weights_to_fp8(w, cols)[0].cpu().double()


def norm64(x, w, eps=1e-6):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.cpu().double()


def layer64(x, p, heads, kv_heads, dim, inner, window):
    """One sequence [tokens, hidden] -> the layer's output."""
    t, hidden = x.shape
    qkv = (norm64(x, p["norm1"]) @ exact_weights(p["qkv"], hidden).T).view(t, -1, dim)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], dim=1)
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


def build(seed, layers, hidden, heads, kv_heads, dim, inner, dtype, batch, tokens, page, window):
    from paper_1905_13298_amd import decoder
    rng = np.random.default_rng(seed)
    ps = [layer_params(rng, hidden, heads, kv_heads, dim, inner, dtype) for _ in range(layers)]
    norm = torch.from_numpy(1 + 0.2 * rng.standard_normal(hidden)).to(DEV, dtype)
    make = lambda: decoder.Decoder([decoder.DecoderLayer(p, heads, kv_heads, dim, inner, window=window) for p in ps],  # noqa: E731
                                   norm, batch, tokens, page)
    return make, ps, norm, rng


@pytest.mark.parametrize("layers,hidden,heads,kv_heads,dim,inner,dtype,page,window", [
    (1, 256, 8, 2, 32, 512, BF16, 16, 0),
    (2, 200, 5, 5, 48, 330, F16, 32, 0),
    (2, 512, 8, 1, 128, 1024, BF16, 64, 24),
])
def test_decoder(layers, hidden, heads, kv_heads, dim, inner, dtype, page, window):
    batch, prompt, single = 3, 70, 5
    make, ps, norm, rng = build(1, layers, hidden, heads, kv_heads, dim, inner, dtype, batch, prompt + single, page, window)
    x = torch.from_numpy(rng.standard_normal((batch, prompt + single, hidden))).to(dtype)
    counts = torch.tensor([prompt, 1, 33])
    model = make()
    first = model(x[:, :prompt].to(DEV), counts.int().to(DEV))
    steps = [model(x[:, prompt + i:prompt + i + 1].to(DEV)) for i in range(single)]
    assert model.length.tolist() == (counts + single).tolist()
    bound = 2.0 ** -4 * math.sqrt(5 * layers)
    for b in range(batch):
        n = int(counts[b])
        y = torch.cat([x[b, :n], x[b, prompt:]]).double()
        for p in ps:
            y = layer64(y, p, heads, kv_heads, dim, inner, window)
        y = norm64(y, norm)
        got = torch.cat([first[b, :n]] + [s[b] for s in steps]).cpu().double()
        for part in (slice(0, n), slice(n, n + single)):
            err = (got[part] - y[part]).square().mean().sqrt() / y[part].square().mean().sqrt()
            assert err <= bound, (b, part, float(err), bound)


def test_decoder_graph_and_reset():
    make, _, _, rng = build(2, 2, 256, 8, 2, 64, 512, BF16, 2, 64, 16, 0)
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


@pytest.mark.parametrize("m,hidden,n,dtype", [(1, 256, 128, BF16), (100, 200, 330, F16), (300, 1000, 520, BF16)])
def test_norm_linear_backward(m, hidden, n, dtype):
    from paper_1905_13298_amd import decoder
    rng = np.random.default_rng(3)
    w = shift_codes(rng, n, hidden)
    norm = torch.from_numpy(1 + 0.2 * rng.standard_normal(hidden)).to(DEV, dtype)
    make = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(DEV, dtype)  # noqa: E731
    x, r, dy, dh = make(m, hidden), make(m, hidden), make(m, n), make(m, hidden)
    part = decoder.NormLinear(norm, *decoder.weights(w, hidden))
    y, h, rstd = part(x, r)
    dx, dw = part.backward(dy, h, rstd, dh)
    h64 = h.cpu().double().requires_grad_()
    n64 = norm.cpu().double().requires_grad_()
    out = h64 / torch.sqrt((h64 * h64).mean(-1, keepdim=True) + 1e-6) * n64 @ exact_weights(w, hidden).T
    ((out * dy.cpu().double()).sum() + (h64 * dh.cpu().double()).sum()).backward()
    for got, want in ((y, out.detach()), (dx, h64.grad), (dw, n64.grad)):
        err = (got.cpu().double() - want).square().mean().sqrt() / want.square().mean().sqrt()
        assert err <= 2.0 ** -4, float(err)


def test_decoder_refuses():
    from paper_1905_13298_amd import decoder
    p = layer_params(np.random.default_rng(4), 64, 4, 2, 16, 128, BF16)
    with pytest.raises(ValueError, match="query heads"):
        decoder.DecoderLayer(p, 4, 3, 16, 128)
    with pytest.raises(ValueError, match="qkv must have"):
        decoder.DecoderLayer(p, 4, 1, 16, 128)
    with pytest.raises(ValueError, match="words a row"):
        decoder.weights(p["out"], 128)
    with pytest.raises(ValueError, match="columns"):
        decoder.weights(torch.zeros(4, 8), 16)
