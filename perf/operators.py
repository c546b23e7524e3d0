"""The 8-bit operators of a language model's decoder layer, as measurable cases.

What a layer with 8-bit weights, activations and cache runs for its tokens: the
root-mean-square norm with the residual's addition and an 8-bit output (and its
gradient), the quantiser of an activation with or without a SiLU gate, the product
of 8-bit matrices (and its input gradient), the append to a paged 8-bit cache of keys
and values, and the attention that reads it. Every 8-bit number is a float8 (E4M3, or
E5M2 for weights that are signed powers of two) with a power-of-two scale (E8M0): one
for each 128 elements of an activation's row, for each 128 x 128 elements of a weight
matrix, and for each page of tokens and head of a cache.

`own` chooses between the plain forms (elementary torch operations in 32 bits) and the
calls of ``paper_1905_13298_amd.ops``. Sizes are generic ones and those of the project's
own classifiers (4096 -> 4096, 2048 -> 1000). Activations are normal with a few large
channels, weights normal with the spread of a layer's, keys and values normal with a
spread from token to token.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0" if torch.cuda.is_available() else "cpu"
BLOCK = 128
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
CACHE_RANGE = 48             # a cache's scales are 2^-48 .. 2^48


def _norm(name, rows, cols, **kw):
    return dict(name=name, kind="norm", rows=rows, cols=cols, type="bf16", residual=True, quantize=True) | kw


def _quant(name, rows, cols, **kw):
    return dict(name=name, kind="quant", rows=rows, cols=cols, type="bf16", gate=True) | kw


def _product(name, m, n, k, **kw):
    return dict(name=name, kind="product", m=m, n=n, k=k, weights="e4m3", out="bf16") | kw


def _append(name, batch, tokens, before, **kw):
    return dict(name=name, kind="append", batch=batch, tokens=tokens, before=before, heads=8, dim=128, page=64,
                type="bf16") | kw


def _attention(name, batch, tokens, longest, **kw):
    return dict(name=name, kind="attention", batch=batch, tokens=tokens, longest=longest, heads=8, group=4, dim=128,
                page=64, window=0, type="bf16", even=False) | kw


def listed():
    return [
        # Before a layer's first product, one token of each of 8 sequences: all latency.
        _norm("norm_8x4096", 8, 4096),
        # The norm's gradient over a training batch's tokens: one pass over four large tensors.
        _norm("norm_grad_8192x4096", 8192, 4096, kind="norm_grad"),
        # A gated MLP's activation for 16 tokens being decoded, into the 8-bit input of the next product.
        _quant("gate_16x8192", 16, 8192),
        # The same over a long prompt, with a ragged width (85 blocks and 120 elements).
        _quant("gate_4099x11000", 4099, 11000),
        # Eight tokens through a square layer with shift weights: reading the weights.
        _product("product_8x4096x4096", 8, 4096, 4096, weights="e5m2"),
        # A prompt's tokens through a wide layer: the matrix cores' rate.
        _product("product_8192x8192x4096", 8192, 8192, 4096),
        # The input gradient of a 2048 -> 1000 classifier over an odd number of tokens.
        _product("product_grad_2005x1000x2048", 2005, 1000, 2048, kind="product_grad"),
        # One new token for each of 64 sequences: single vectors into pages that are part full.
        _append("append_64x1", 64, 1, 1000),
        # Four prompts of about 2000 tokens into new pages: streaming.
        _append("append_4x2001", 4, 2001, 0),
        # One sequence with a long context, one new token: few rows, a long axis.
        _attention("attention_1x1_131072", 1, 1, 131072, even=True),
        # A serving batch of 48 sequences of very different lengths, one token each.
        _attention("attention_48x1_8192", 48, 1, 8192),
        # Two prompts' chunks of 1000 tokens on top of up to 7000 cached ones.
        _attention("attention_2x1000_8000", 2, 1000, 8000, even=True),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size spread over its logarithm: as it falls, or a multiple of 16 or 128."""
    v, by = _logint(rng, lo, hi), rng.choice([1, 16, 128])
    return min(hi, max(lo, (v + by - 1) // by * by))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "quant", "product", "product", "product_grad", "append", "attention",
                       "attention", "attention"])
    kw = dict(kind=kind, type=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if kind in ("norm", "norm_grad", "quant"):
        kw.update(rows=_logint(rng, 1, 8192), cols=_size(rng, 32, 12288))
        if kind == "quant":
            return _quant("", **kw | dict(gate=rng.random() < 0.6))
        return _norm("", **kw | dict(residual=rng.random() < 0.7, quantize=kind == "norm" and rng.random() < 0.7))
    if kind in ("product", "product_grad"):
        return _product("", _logint(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 64, 4096), kind=kind,
                        weights=rng.choice(["e4m3", "e5m2"]), out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    heads, dim, page = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 128, 128, 256]), rng.choice([16, 32, 64, 128])
    if kind == "append":
        tokens = rng.choice([1, 1, _logint(rng, 2, 2048)])
        batch = _logint(rng, 1, max(1, min(64, 16384 // tokens)))
        return _append("", batch, tokens, rng.choice([0, _logint(rng, 1, 1024)]), heads=heads, dim=dim, page=page,
                       type=kw["type"])
    tokens = rng.choice([1, 1, 1, rng.randint(2, 8), _logint(rng, 9, 1024)])
    group = rng.choice([1, 2, 4, 7, 8])
    while True:
        batch, longest = _logint(rng, 1, 64), _logint(rng, 1, 131072)
        longest = max(longest, tokens)
        if batch * longest * heads * dim <= 200e6 and batch * heads * group * tokens * longest * dim <= 60e9:
            break
    return _attention("", batch, tokens, longest, heads=heads, group=group, dim=dim, page=page, even=rng.random() < 0.3,
                      window=rng.choice([0, 0, 0, _logint(rng, 16, 8192)]), type=rng.choice(["bf16", "bf16", "f16"]))


# ---------------------------------------------------------------------------
# Inputs.


class _Draw:
    """Random tensors on the device from one seed."""

    def __init__(self, seed):
        self.g = torch.Generator(DEV)
        self.g.manual_seed(int(seed))

    def normal(self, *shape, std=1.0):
        return torch.randn(shape, generator=self.g, device=DEV) * std

    def uniform(self, *shape, lo=0.0, hi=1.0):
        return torch.rand(shape, generator=self.g, device=DEV) * (hi - lo) + lo

    def integers(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device=DEV, dtype=torch.int32)

    def order(self, n):
        return torch.randperm(n, generator=self.g, device=DEV).to(torch.int32)

    def activations(self, rows, cols, std=1.0):
        """Normal, with one channel in 64 eight times as large."""
        return self.normal(rows, cols, std=std) * torch.where(self.uniform(cols) < 1 / 64, 8.0, 1.0)


def _exponent(amax, lo=1, hi=254, zero=127):
    """The E8M0 byte of the least power of two that brings amax to at most 448 (`zero` where amax is 0)."""
    e = ((amax.contiguous().view(torch.int32) + 0x1FFFFF) >> 23) - 8
    return torch.where(amax == 0, zero, e.clamp(lo, hi))


def _power(e):
    """2^(e - 127) in 32 bits, for e in 1 .. 254."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def _scales(e):
    return e.to(torch.uint8).view(E8M0)


def _rows16(x8):
    """x8 with rows that begin on 16 bytes, as the quantisers lay them out."""
    rows, cols = x8.shape
    out = torch.zeros(rows, (cols + 15) // 16 * 16, dtype=torch.uint8, device=x8.device).view(x8.dtype)
    out.view(torch.uint8)[:, :cols] = x8.view(torch.uint8)
    return out[:, :cols]


def _blocks(y, rows=1):
    """y [r, c] as [r / rows, rows, c / 128, 128], filled up with zeros."""
    r, c = y.shape
    y = torch.nn.functional.pad(y, (0, -c % BLOCK, 0, -r % rows))
    return y.reshape(y.shape[0] // rows, rows, y.shape[1] // BLOCK, BLOCK)


def _to_blocks8(y, rows=1, to=E4M3):
    """(8-bit y, its scales): a scale for each `rows` x 128 elements."""
    r, c = y.shape
    b = _blocks(y, rows)
    size = torch.where(torch.isfinite(b), b.abs(), 0.0).amax((1, 3))
    e = _exponent(size)
    b = b * _power(254 - e)[:, None, :, None]
    return b.reshape(-1, b.shape[2] * BLOCK)[:r, :c].to(to), _scales(e)


def prepare(case, seed):
    return {"case": case} | _PREPARE[case["kind"]](case, _Draw(seed))


def _prepare_norm(case, d):
    rows, cols, t = case["rows"], case["cols"], TYPES[case["type"]]
    s = {"x": d.activations(rows, cols).to(t), "weight": d.normal(cols, std=0.2).add(1).to(t),
         "residual": d.activations(rows, cols, std=3).to(t) if case["residual"] else None}
    return s


def _prepare_norm_grad(case, d):
    rows, cols, t = case["rows"], case["cols"], TYPES[case["type"]]
    h = d.activations(rows, cols, std=3).to(t)
    return {"h": h, "weight": d.normal(cols, std=0.2).add(1).to(t), "dy": d.normal(rows, cols).to(t),
            "dh": d.normal(rows, cols).to(t) if case["residual"] else None,
            "rstd": (h.float().square().mean(1) + 1e-6).rsqrt()}


def _prepare_quant(case, d):
    rows, cols, t = case["rows"], case["cols"], TYPES[case["type"]]
    if not case["gate"]:
        return {"x": d.activations(rows, cols).to(t), "gate": None}
    both = torch.cat([d.normal(rows, cols), d.activations(rows, cols)], 1).to(t)   # one product's two halves
    return {"x": both[:, cols:], "gate": both[:, :cols]}


def _prepare_product(case, d):
    m, n, k = case["m"], case["n"], case["k"]
    grad = case["kind"] == "product_grad"
    if case["weights"] == "e5m2":   # signed powers of two, 2^0 .. 2^-14, a tenth of them zero
        p = torch.exp2(-d.integers(0, 15, n, k).float())
        w8 = torch.where(d.uniform(n, k) < 0.1, 0.0, torch.where(d.uniform(n, k) < 0.5, -p, p)).to(E5M2)
        ws = _scales(torch.full(((n + BLOCK - 1) // BLOCK, (k + BLOCK - 1) // BLOCK), 127, device=DEV))
    else:
        w8, ws = _to_blocks8(d.normal(n, k, std=0.02), BLOCK)
    x8, xs = _to_blocks8(d.normal(m, n, std=1e-3) if grad else d.activations(m, k))
    return {"x8": _rows16(x8), "xs": xs, "w8": _rows16(w8), "ws": ws}


def _pages(d, needed, columns, pages=None):
    """A table [sequence, column] of pages in random order, -1 past each sequence's last, and how many pages there are
    (`pages`, or what is needed and three more)."""
    last = torch.cumsum(needed, 0)
    pool = d.order(pages or int(last[-1]) + 3)
    at = (last - needed)[:, None] + torch.arange(columns, device=DEV)[None, :]
    inside = torch.arange(columns, device=DEV)[None, :] < needed[:, None]
    return torch.where(inside, pool[at.clamp(max=pool.numel() - 1)], -1).to(torch.int32), pool.numel()


def _page8(x):
    """Pages [p, h, a, b] in 8 bits, and their scales [p, h]."""
    e = _exponent(x.abs().amax((2, 3)), 127 - CACHE_RANGE, 127 + CACHE_RANGE, 127 - CACHE_RANGE)
    return (x * _power(254 - e)[:, :, None, None]).to(E4M3), _scales(e)


def _cache(d, pages, heads, page, dim):
    k8, ks = _page8(d.normal(pages, heads, page, dim) * d.uniform(pages, heads, page, 1, lo=0.5, hi=2.0))
    v8, vs = _page8(d.normal(pages, heads, dim, page) * d.uniform(pages, heads, 1, page, lo=0.1, hi=1.5))
    return {"k_cache": k8, "v_cache": v8, "k_scales": ks, "v_scales": vs}


def _prepare_append(case, d):
    b, t, before, page = case["batch"], case["tokens"], case["before"], case["page"]
    start = d.integers(before // 2, before + 1, b)
    columns = (before + t + page - 1) // page + 1
    table, pages = _pages(d, (start + t + page - 1) // page, columns, b * columns + 3)
    kv = TYPES[case["type"]]
    s = _cache(d, pages, case["heads"], page, case["dim"])
    s["k"] = (d.normal(b, t, case["heads"], case["dim"]) * d.uniform(b, t, 1, 1, lo=0.5, hi=3.0)).to(kv)
    s["v"] = (d.normal(b, t, case["heads"], case["dim"]) * d.uniform(b, t, 1, 1, lo=0.1, hi=2.0)).to(kv)
    return s | {"table": table, "start": start}


def _prepare_attention(case, d):
    b, t, longest, page = case["batch"], case["tokens"], case["longest"], case["page"]
    length = d.integers(0 if b > 3 else max(1, longest // 2), longest + 1, b)
    length[0] = longest
    if case["even"]:
        length = torch.clamp(length, min=longest * 7 // 8)
    columns = (longest + page - 1) // page
    table, pages = _pages(d, (length + page - 1) // page, columns)
    s = _cache(d, pages, case["heads"], page, case["dim"])
    q = d.normal(b, t, case["heads"] * case["group"], case["dim"]).to(TYPES[case["type"]])
    return s | {"q": q, "table": table, "length": length, "count": torch.clamp(length, max=t)}


_PREPARE = {"norm": _prepare_norm, "norm_grad": _prepare_norm_grad, "quant": _prepare_quant,
            "product": _prepare_product, "product_grad": _prepare_product, "append": _prepare_append,
            "attention": _prepare_attention}


# ---------------------------------------------------------------------------
# One pass.


def run(state):
    kind = state["case"]["kind"]
    return (_OWN if own else _PLAIN)[kind](state)


def _plain_norm(s):
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
    f = h.float()
    rstd = 1 / torch.sqrt(f.square().mean(1) + 1e-6)
    y = f * rstd[:, None] * s["weight"].float()
    if s["case"]["quantize"]:
        return (*_to_blocks8(y), h, rstd)
    return y.to(h.dtype), h, rstd


def _plain_norm_grad(s):
    h, dy, r = s["h"].float(), s["dy"].float(), s["rstd"][:, None]
    n = h * r
    g = dy * s["weight"].float()
    dx = r * (g - n * (g * n).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return dx.to(s["h"].dtype), (dy * n).sum(0).to(s["weight"].dtype)


def _plain_quant(s):
    y = s["x"].float()
    if s["gate"] is not None:
        g = s["gate"].float()
        y = g / (1 + torch.exp(-g)) * y
    return _to_blocks8(y)


def _values(x8, scales, rows=1):
    r, c = x8.shape
    s = _power(scales.view(torch.uint8))
    return x8.float() * s.repeat_interleave(rows, 0)[:r].repeat_interleave(BLOCK, 1)[:, :c]


def _plain_product(s):
    x, w = _values(s["x8"], s["xs"]), _values(s["w8"], s["ws"], BLOCK)
    return (x @ (w if s["case"]["kind"] == "product_grad" else w.t())).to(TYPES[s["case"]["out"]])


def _plain_append_to(cache, scales, new, s, tokens_last):
    """New tokens [b, t, h, d] into the pages of one cache: what is held there is rounded again where a scale grows."""
    b, t = new.shape[:2]
    page = s["case"]["page"]
    start = s["start"].long()
    touched = (t + page - 2) // page + 1
    first = start // page
    col = first[:, None] + torch.arange(touched, device=new.device)                        # [b, touched]
    at = col[:, :, None] * page + torch.arange(page, device=new.device)                    # position of each slot
    fresh = (at >= start[:, None, None]) & (at < start[:, None, None] + t)
    older = at < start[:, None, None]
    pid = s["table"].long().gather(1, col.clamp(max=s["table"].shape[1] - 1))
    used = fresh.any(2) & (col < s["table"].shape[1])
    pid = pid.clamp(min=0)
    x = new.float()[torch.arange(b, device=new.device)[:, None, None], (at - start[:, None, None]).clamp(0, t - 1)]
    x = x.transpose(2, 3)                                                                  # [b, touched, h, page, d]
    fresh, older = fresh[:, :, None, :, None], older[:, :, None, :, None]
    size = torch.where(fresh & torch.isfinite(x), x.abs(), 0.0).amax((3, 4))
    lowest = 127 - CACHE_RANGE
    e = _exponent(size, lowest, 127 + CACHE_RANGE, lowest)
    before = scales.view(torch.uint8)[pid].to(torch.int32)                                 # [b, touched, h]
    e = torch.where(older.any(3)[..., 0], torch.maximum(e, before), e)
    old = cache[pid]
    if tokens_last:
        old = old.view(torch.uint8).transpose(3, 4).contiguous().view(E4M3)
    kept = old.float() * _power(127 + before - e)[..., None, None]
    y = torch.where(fresh, x * _power(254 - e)[..., None, None], kept)
    y = torch.where(torch.isfinite(y), y.clamp(-448, 448), math.nan).to(E4M3).view(torch.uint8)
    y = torch.where(fresh | older, y, old.view(torch.uint8))
    if tokens_last:
        y = y.transpose(3, 4)
    cache.view(torch.uint8)[pid[used]] = y[used]
    scales.view(torch.uint8)[pid[used]] = e[used].to(torch.uint8)


def _plain_append(s):
    _plain_append_to(s["k_cache"], s["k_scales"], s["k"], s, False)
    _plain_append_to(s["v_cache"], s["v_scales"], s["v"], s, True)
    return s["k_cache"], s["k_scales"], s["v_cache"], s["v_scales"]


def _plain_attention(s):
    case = s["case"]
    b, t, hq, dim = s["q"].shape
    heads, group, page = case["heads"], case["group"], case["page"]
    pid = s["table"].long().clamp(min=0)
    keys = s["k_cache"][pid].float() * _power(s["k_scales"].view(torch.uint8)[pid])[..., None, None]
    keys = keys.permute(0, 2, 4, 1, 3).reshape(b, heads, dim, -1)
    q = s["q"].float().reshape(b, t, heads, group, dim).permute(0, 2, 1, 3, 4).reshape(b, heads, t * group, dim)
    w = (q @ keys / math.sqrt(dim)).reshape(b, heads, t, group, -1)
    del keys
    where = s["length"][:, None] - s["count"][:, None] + torch.arange(t, device=q.device)[None, :]
    j = torch.arange(w.shape[-1], device=q.device)
    seen = (j <= where[..., None]) & (torch.arange(t, device=q.device)[None, :, None] < s["count"][:, None, None])
    if case["window"]:
        seen &= j > where[..., None] - case["window"]
    seen = seen[:, None, :, None, :]
    w = torch.where(seen, w, -math.inf)
    top = w.amax(-1, keepdim=True)
    w = torch.exp(w - torch.where(torch.isfinite(top), top, 0.0))
    total = w.sum(-1, keepdim=True)
    values = s["v_cache"][pid].float() * _power(s["v_scales"].view(torch.uint8)[pid])[..., None, None]
    values = values.permute(0, 2, 1, 4, 3).reshape(b, heads, -1, dim)
    o = (w.reshape(b, heads, t * group, -1) @ values).reshape(b, heads, t, group, dim)
    o = torch.where(total > 0, o / total, 0.0)
    return o.permute(0, 2, 1, 3, 4).reshape(b, t, hq, dim).to(s["q"].dtype)


_PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "quant": _plain_quant, "product": _plain_product,
          "product_grad": _plain_product, "append": _plain_append, "attention": _plain_attention}


def _own_norm(s):
    from paper_1905_13298_amd import ops
    y, scales, h, rstd = ops.rms_norm(s["x"], s["weight"], s["residual"], eps=1e-6, quantize=s["case"]["quantize"])
    return (y, h, rstd) if scales is None else (y, scales, h, rstd)


def _own_norm_grad(s):
    from paper_1905_13298_amd import ops
    return ops.rms_norm_backward(s["dy"], s["h"], s["weight"], s["rstd"], s["dh"])


def _own_quant(s):
    from paper_1905_13298_amd import ops
    return ops.quantize_fp8(s["x"], s["gate"])


def _own_product(s):
    from paper_1905_13298_amd import ops
    call = ops.linear_fp8_backward_data if s["case"]["kind"] == "product_grad" else ops.linear_fp8
    return call(s["x8"], s["xs"], s["w8"], s["ws"], out_dtype=TYPES[s["case"]["out"]])


def _own_append(s):
    from paper_1905_13298_amd import ops
    ops.kv_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"], s["table"], s["start"])
    return s["k_cache"], s["k_scales"], s["v_cache"], s["v_scales"]


def _own_attention(s):
    from paper_1905_13298_amd import ops
    return ops.attention_fp8(s["q"], s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"], s["table"], s["length"],
                             count=s["count"], window=s["case"]["window"])


_OWN = {"norm": _own_norm, "norm_grad": _own_norm_grad, "quant": _own_quant, "product": _own_product,
        "product_grad": _own_product, "append": _own_append, "attention": _own_attention}


# ---------------------------------------------------------------------------
# What a pass cannot do without.


def _lengths(case):
    """The expected sum of the lengths of a case's sequences."""
    b, longest = case["batch"], case["longest"]
    low = longest * 7 / 8 if case["even"] else 0 if b > 3 else max(1, longest // 2)
    rest = (low + longest) / 2 if not case["even"] or b <= 3 else low + longest / 128
    return longest + (b - 1) * rest


def work(case):
    kind = case["kind"]
    size = {"bf16": 2, "f16": 2, "f32": 4}
    if kind in ("norm", "norm_grad", "quant"):
        n, e = case["rows"] * case["cols"], size[case["type"]]
        if kind == "quant":
            return {"bytes": n * (e * (2 if case["gate"] else 1) + 1 + 1 / BLOCK), "flops": n * (6 if case["gate"] else 2)}
        if kind == "norm":
            out = 1 + 1 / BLOCK if case["quantize"] else e
            return {"bytes": n * (e * (3 if case["residual"] else 1) + out) + case["cols"] * e, "flops": 6 * n}
        return {"bytes": n * e * (4 if case["residual"] else 3) + 2 * case["cols"] * e, "flops": 10 * n}
    if kind in ("product", "product_grad"):
        m, n, k = case["m"], case["n"], case["k"]
        a, c = (n, k) if kind == "product_grad" else (k, n)
        return {"bytes": m * a * (1 + 1 / BLOCK) + n * k + m * c * size[case["out"]], "flops": 2 * m * n * k}
    if kind == "append":
        new = 2 * case["batch"] * case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": new * (size[case["type"]] + 1), "flops": 2 * new}
    total, rows = _lengths(case), case["batch"] * case["tokens"] * case["heads"] * case["group"]
    mean = total / case["batch"]
    seen = max(1.0, mean - (min(mean, case["tokens"]) - 1) / 2)
    kept = mean
    if case["window"]:
        seen, kept = min(seen, case["window"]), min(mean, case["window"] + case["tokens"])
    return {"bytes": 2 * case["batch"] * kept * case["heads"] * case["dim"] + 2 * rows * case["dim"] * size[case["type"]],
            "flops": 4 * rows * seen * case["dim"]}


# ---------------------------------------------------------------------------
# The definitions in 64 bits, one row, head or page at a time.


def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed))


def _least_scale(largest):
    """The least power of two that brings `largest` (64 bits, > 0) to at most 448."""
    return torch.exp2(torch.ceil(torch.log2(largest / 448)))


def _exact_blocks(y):
    """Each element over its block's scale, and the scales."""
    over, scales = torch.empty_like(y), []
    for c in range(0, y.shape[1], 128):
        part = y[:, c:c + 128]
        largest = part.abs().max(1).values
        s = torch.where(largest > 0, _least_scale(torch.where(largest > 0, largest, 448.0)), 1.0)
        scales.append(s)
        over[:, c:c + 128] = part / s[:, None]
    return over, torch.stack(scales, 1)


def _exact_norm(case, s):
    h = s["x"].double()
    if case["residual"]:
        h = h + s["residual"].double()
    stored = h.to(s["x"].dtype).double()       # the sum as it is kept: what is normed
    rstd = torch.pow(torch.sum(stored * stored, 1) / case["cols"] + 1e-6, -0.5)
    y = stored * s["weight"].double()[None, :] * rstd[:, None]
    return (*_exact_blocks(y), h, rstd) if case["quantize"] else (y, h, rstd)


def _exact_norm_grad(case, s):
    h, w, r, dy = (s[n].double() for n in ("h", "weight", "rstd", "dy"))
    inner = torch.sum(dy * w * h, 1)
    dx = dy * w * r[:, None] - h * (r.pow(3) * inner / case["cols"])[:, None]
    if case["residual"]:
        dx += s["dh"].double()
    return dx, torch.sum(dy * h * r[:, None], 0)


def _exact_quant(case, s):
    y = s["x"].double()
    if case["gate"]:
        y = y * s["gate"].double() * torch.sigmoid(s["gate"].double())
    return _exact_blocks(y)


def _exact_product(case, s):
    x, w = s["x8"].double(), s["w8"].double()
    xs, ws = s["xs"].double(), s["ws"].double()
    for j in range(xs.shape[1]):
        x[:, 128 * j:128 * j + 128] *= xs[:, j:j + 1]
    for i in range(ws.shape[0]):
        for j in range(ws.shape[1]):
            w[128 * i:128 * i + 128, 128 * j:128 * j + 128] *= ws[i, j]
    return torch.mm(x, w) if case["kind"] == "product_grad" else torch.mm(x, w.t().contiguous())


def _exact_append(case, s):
    page, t = case["page"], case["tokens"]
    got = []
    for name, last in (("k", False), ("v", True)):
        cache, scales, new = s[name + "_cache"].double(), s[name + "_scales"].double(), s[name].double()
        table, start = s["table"].cpu().tolist(), s["start"].cpu().tolist()
        if case["batch"] * (t // page + 2) > 20000:
            return None
        for b, (row, first) in enumerate(zip(table, start)):
            for c in range(first // page, (first + t - 1) // page + 1):
                lo, hi = max(first, c * page), min(first + t, c * page + page)
                x = new[b, lo - first:hi - first].transpose(0, 1)                     # [h, tokens, d]
                largest = x.abs().amax((1, 2))
                scale = _least_scale(largest.clamp(min=1e-300)).clamp(2.0 ** -CACHE_RANGE, 2.0 ** CACHE_RANGE)
                held = cache[row[c]].transpose(1, 2) if last else cache[row[c]]       # [h, page, d], changed in place
                if lo > c * page:
                    grown = torch.maximum(scale, scales[row[c]])
                    held[:, :lo - c * page] *= (scales[row[c]] / grown)[:, None, None]
                    scale = grown
                held[:, lo - c * page:hi - c * page] = (x / scale[:, None, None]).clamp(-448, 448)
                scales[row[c]] = scale
        got += [cache, scales]
    return tuple(got)


def _exact_attention(case, s):
    b, t, hq, dim = s["q"].shape
    length, count = s["length"].cpu().tolist(), s["count"].cpu().tolist()
    if b * hq > 4096:
        return None
    out = torch.zeros(b, t, hq, dim, dtype=torch.float64, device=s["q"].device)
    for i in range(b):
        n, c = length[i], count[i]
        if n == 0:
            continue
        rows = s["table"][i, :(n - 1) // case["page"] + 1].long()
        for h in range(case["heads"]):
            k = s["k_cache"][rows, h].double() * s["k_scales"][rows, h].double()[:, None, None]
            v = s["v_cache"][rows, h].double() * s["v_scales"][rows, h].double()[:, None, None]
            k = k.reshape(-1, dim)[:n].t().contiguous()
            v = v.transpose(1, 2).reshape(-1, dim)[:n].contiguous()
            own_place = torch.arange(n - c, n, device=k.device)[:, None]
            other = torch.arange(n, device=k.device)[None, :]
            hidden = other > own_place
            if case["window"]:
                hidden |= other <= own_place - case["window"]
            for g in range(case["group"]):
                q = s["q"][i, :c, h * case["group"] + g].double()
                p = torch.softmax(torch.mm(q, k).mul_(dim ** -0.5).masked_fill_(hidden, -math.inf), 1)
                out[i, :c, h * case["group"] + g] = torch.mm(p, v)
    return out


_EXACT = {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "quant": _exact_quant, "product": _exact_product,
          "product_grad": _exact_product, "append": _exact_append, "attention": _exact_attention}
