"""Rotated heads and a 4-bit cache of a language model's decoder layer, as measurable cases.

What stands in a layer between the product that forms queries, keys and values and the
attention's output, where the model has positions and its cache is to hold long contexts: the
root-mean-square norm of each query and key head with the rotation by its token's position
in the same pass (one axis, or several for pictures and video) and its gradient, the append to a
paged cache in 4 bits, the way back to floats, and the attention that reads the cache. A 4-bit number
is an E2M1 float (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), with a power-of-two scale (E8M0) for
each 32 elements of a token's head.

`own` chooses between the plain forms (elementary torch operations in 32 bits, angles in 64) and
the calls of ``paper_1905_13298_amd.ops``. Sizes are generic. Queries and keys before the norm are
normal with a few large channels, as parts of one product's rows; keys and values for the cache are
normal with a spread from token to token.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0" if torch.cuda.is_available() else "cpu"
BLOCK = 32                   # elements of a token's head that share a scale
LOW, HIGH = 127 - 23, 127 + 13      # scale bytes of a cache: every number that it holds is a 16-bit float
NAN = 255                    # the scale byte of a block with an element that is no finite number
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _rotary(name, batch, tokens, **kw):
    return dict(name=name, kind="rotary", batch=batch, tokens=tokens, heads=32, kv_heads=8, dim=128, pairs=64, axes=1, norm=True,
                interleaved=False, far=8192, theta=1e4, type="bf16") | kw


def _append(name, batch, tokens, before, **kw):
    return dict(name=name, kind="append", batch=batch, tokens=tokens, before=before, heads=8, dim=128, page=64, type="bf16") | kw


def _read(name, batch, longest, **kw):
    return dict(name=name, kind="read", batch=batch, longest=longest, heads=8, dim=128, page=64, type="bf16") | kw


def _attention(name, batch, tokens, longest, **kw):
    return dict(name=name, kind="attention", batch=batch, tokens=tokens, longest=longest, heads=8, group=4, dim=128,
                page=64, window=0, type="bf16", even=False) | kw


def listed():
    return [
        # One token of each of 8 sequences, far into their contexts: all latency.
        _rotary("rotary_8x1", 8, 1, far=131072, theta=5e5),
        # Four prompts of 2001 tokens: one pass over queries and keys.
        _rotary("rotary_4x2001", 4, 2001),
        # Two videos' patches with positions in time, height and width, neighbouring elements as pairs, no norm, an odd
        # count and a head size that is no power of two.
        _rotary("rotary_axes_2x1221", 2, 1221, heads=16, kv_heads=16, dim=80, pairs=40, axes=3, norm=False, interleaved=True,
                far=64, type="f16"),
        # The gradient over a training batch of 4 x 2048 tokens.
        _rotary("rotary_grad_4x2048", 4, 2048, kind="rotary_grad"),
        # The same in 32 bits, with a quarter of each head left without positions, over ragged sizes.
        _rotary("rotary_grad_3x333", 3, 333, kind="rotary_grad", heads=12, kv_heads=4, dim=96, pairs=36, type="f32"),
        # One new token for each of 64 sequences, into pages that are part full, and back.
        _append("append_64x1", 64, 1, 1000),
        # Four prompts of 2001 tokens, and back.
        _append("append_4x2001", 4, 2001, 0),
        # The first 20000 or so tokens of six sequences as floats, for a pass that wants them so.
        _read("read_6x20000", 6, 20000),
        # One sequence with a long context, one new token: few rows, a long axis.
        _attention("attention_1x1_131072", 1, 1, 131072, even=True),
        # A serving batch of 48 sequences of very different lengths, one token each.
        _attention("attention_48x1_8192", 48, 1, 8192),
        # Chunks of 1000 tokens of two prompts, on top of up to 7000 cached ones.
        _attention("attention_2x1000_8000", 2, 1000, 8000, even=True),
        # Five sequences with 3 drafted tokens each to be looked over, a window, small pages and an odd head size.
        _attention("attention_5x3_4000", 5, 3, 4000, heads=4, group=7, dim=80, page=16, window=1500, type="f16"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "rotary_grad", "rotary_grad", "append", "append", "read", "attention", "attention", "attention"])
    kw = dict(kind=kind, type=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if kind in ("rotary", "rotary_grad"):
        dim = rng.choice([32, 64, 80, 96, 128, 128, 192, 256])
        heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4, 7])
        vectors = 200000 * 128 // dim // (heads * (group + 1))
        tokens = rng.choice([1, _logint(rng, 1, min(4096, vectors))])
        return _rotary("", _logint(rng, 1, max(1, min(64, vectors // tokens))), tokens, heads=heads * group, kv_heads=heads, dim=dim,
                       pairs=rng.choice([dim // 2, dim // 2, dim // 4, rng.randint(3, dim // 2)]), axes=rng.choice([1, 1, 2, 3]),
                       norm=rng.random() < 0.7, interleaved=rng.random() < 0.3, far=_logint(rng, 16, 1 << 20),
                       theta=rng.choice([1e4, 5e5]), **kw)
    heads, dim, page = rng.choice([1, 2, 4, 8]), rng.choice([32, 64, 80, 96, 128, 128, 256]), rng.choice([16, 32, 64, 128])
    kw.update(heads=heads, dim=dim, page=page)
    if kind == "append":
        tokens = rng.choice([1, 1, _logint(rng, 2, 2048)])
        batch = _logint(rng, 1, max(1, min(64, 16384 // tokens)))
        return _append("", batch, tokens, rng.choice([0, _logint(rng, 1, 1024)]), **kw)
    if kind == "read":
        longest = _logint(rng, 1, 20000)
        return _read("", _logint(rng, 1, max(1, min(64, 100000000 // (longest * heads * dim)))), longest, **kw)
    kw["type"] = rng.choice(["bf16", "bf16", "f16"])
    tokens = rng.choice([1, 1, 1, rng.randint(2, 8), _logint(rng, 9, 1024)])
    group = rng.choice([1, 2, 4, 7, 8])
    while True:
        batch, longest = _logint(rng, 1, 64), _logint(rng, 1, 131072)
        longest = max(longest, tokens)
        if batch * longest * heads * dim <= 200e6 and batch * heads * group * tokens * longest * dim <= 60e9:
            break
    return _attention("", batch, tokens, longest, group=group, even=rng.random() < 0.3,
                      window=rng.choice([0, 0, 0, _logint(rng, 16, 8192)]), **kw)


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


def prepare(case, seed):
    return {"case": case} | _PREPARE[case["kind"]](case, _Draw(seed))


def _sections(case):
    """How many pairs go by each axis: the first ones by time, the others evenly by the rest."""
    pairs, axes = case["pairs"], case["axes"]
    if axes == 1:
        return None
    each = pairs // axes
    return tuple([pairs - each * (axes - 1)] + [each] * (axes - 1))


def _frequencies(case):
    """Radians a position for each pair: theta^(-i / pairs)."""
    return torch.pow(torch.tensor(case["theta"], dtype=torch.float64), -torch.arange(case["pairs"], dtype=torch.float64) / case["pairs"]).to(DEV)


def _prepare_rotary(case, d):
    b, t, hq, hk, dim, dtype = case["batch"], case["tokens"], case["heads"], case["kv_heads"], case["dim"], TYPES[case["type"]]
    qkv = d.normal(b, t, hq + 2 * hk, dim) * torch.where(d.uniform(hq + 2 * hk, dim) < 1 / 64, 6.0, 1.0)
    q, k, _ = qkv.to(dtype).split([hq, hk, hk], dim=2)         # the parts of one product's rows
    if case["axes"] == 1:
        start = d.integers(case["far"] // 2, case["far"] + 1, b)
        positions = (start[:, None] + torch.arange(t, device=DEV, dtype=torch.int32)[None, :]).to(torch.int32)
    else:
        # Frames of patches, each sequence's grid of its own width, from a place of its own on.
        wide = d.integers(5, 40, b, 1)
        at = torch.arange(t, device=DEV, dtype=torch.int32)[None, :]
        grid = [torch.div(at, wide * wide, rounding_mode="floor"), torch.div(at, wide, rounding_mode="floor") % wide, at % wide]
        positions = torch.stack([(g + d.integers(0, case["far"] + 1, b, 1)).to(torch.int32) for g in grid[:case["axes"]]])
    s = {"q": q, "k": k, "positions": positions, "frequencies": _frequencies(case), "sections": _sections(case)}
    weight = lambda: d.normal(dim, std=0.2).add(1).to(dtype) if case["norm"] else None  # noqa: E731
    s |= {"q_weight": weight(), "k_weight": weight()}
    if case["kind"] == "rotary_grad":
        s |= {"dq": d.normal(b, t, hq, dim).to(dtype), "dk": d.normal(b, t, hk, dim).to(dtype)}
    return s


def _pages(d, needed, columns, pages=None):
    """A table [sequence, column] of pages in random order, -1 past each sequence's last, and how many pages there are
    (`pages`, or what is needed and three more)."""
    last = torch.cumsum(needed, 0)
    pool = d.order(pages or int(last[-1]) + 3)
    at = (last - needed)[:, None] + torch.arange(columns, device=DEV)[None, :]
    inside = torch.arange(columns, device=DEV)[None, :] < needed[:, None]
    return torch.where(inside, pool[at.clamp(max=pool.numel() - 1)], -1).to(torch.int32), pool.numel()


def _power(e):
    """2^(e - 127) in 32 bits, for e in 1 .. 254."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def _to_4bit(x):
    """x [.., dim] in 32 bits -> (codes [.., dim], a byte each, scale bytes [.., ceil(dim / 32)])."""
    dim = x.shape[-1]
    y = torch.nn.functional.pad(x, (0, -dim % BLOCK))
    y = y.reshape(*y.shape[:-1], -1, BLOCK)
    fine = torch.isfinite(y).all(-1)
    top = torch.where(fine, y.abs().amax(-1), 0.0)
    # The least power of two that brings the largest to 6 = 1.5 * 2^2: a mantissa above 1.5 carries.
    e = (((top.contiguous().view(torch.int32) + 0x3FFFFF) >> 23) - 2).clamp(LOW, HIGH)
    y = torch.where(fine[..., None], y * _power(254 - e)[..., None], 0.0)
    size = y.abs()
    code = torch.zeros(y.shape, dtype=torch.uint8, device=y.device)
    for border, tie_up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (size >= border) if tie_up else (size > border)
    code |= (y < 0).to(torch.uint8) << 3
    return code.reshape(*x.shape[:-1], -1)[..., :dim], torch.where(fine, e, NAN).to(torch.uint8)


def _to_bytes(code):
    """Two codes a byte, the first in the low half."""
    return code[..., 0::2] | code[..., 1::2] << 4


def _page_layout(b, last):
    """Pages [p, h, page, dim / 2] as a cache holds them: keys as they are, values in pieces of 4 tokens x 8 dimensions."""
    if not last:
        return b.contiguous()
    p, h, page, half = b.shape
    return b.reshape(p, h, page // 4, 4, half // 4, 4).transpose(3, 4).contiguous()


def _cache(d, pages, heads, page, dim):
    """A cache of random keys and values (made some pages at a time)."""
    got = {"k_cache": [], "v_cache": [], "k_scales": [], "v_scales": []}
    some = max(1, (1 << 24) // (heads * page * dim))
    for first in range(0, pages, some):
        n = min(some, pages - first)
        for name, last, lo, hi in (("k", False, 0.5, 2.0), ("v", True, 0.1, 1.5)):
            code, e = _to_4bit(d.normal(n, heads, page, dim) * d.uniform(n, heads, page, 1, lo=lo, hi=hi))
            got[name + "_cache"].append(_page_layout(_to_bytes(code), last))
            got[name + "_scales"].append(e.transpose(2, 3))
    got = {name: torch.cat(parts).contiguous() for name, parts in got.items()}
    return got | {name: got[name].view(torch.float8_e8m0fnu) for name in ("k_scales", "v_scales")}


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


def _prepare_read(case, d):
    b, longest, page = case["batch"], case["longest"], case["page"]
    length = d.integers(longest * 3 // 4, longest + 1, b)
    length[0] = longest
    table, pages = _pages(d, (length + page - 1) // page, (longest + page - 1) // page)
    return _cache(d, pages, case["heads"], page, case["dim"]) | {"table": table, "count": length, "start": torch.zeros_like(length)}


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


_PREPARE = {"rotary": _prepare_rotary, "rotary_grad": _prepare_rotary, "append": _prepare_append, "read": _prepare_read,
            "attention": _prepare_attention}


# ---------------------------------------------------------------------------
# One pass.


def run(state):
    kind = state["case"]["kind"]
    return (_OWN if own else _PLAIN)[kind](state)


def _angles(s):
    """(cosines, sines) [batch, tokens, 1, pairs] of a call's pairs, the angles in 64 bits."""
    positions = s["positions"].double()
    if s["sections"] is None:
        a = positions[..., None] * s["frequencies"]
    else:
        parts = torch.split(s["frequencies"], list(s["sections"]))
        a = torch.cat([p[..., None] * f for p, f in zip(positions, parts)], -1)
    return torch.cos(a).float()[:, :, None], torch.sin(a).float()[:, :, None]


def _turn(x, cos, sin, interleaved):
    """Each pair of x turned by its angle."""
    pairs = cos.shape[-1]
    if interleaved:
        a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., 2 * pairs:]], -1)


def _plain_rotary(s):
    cos, sin = _angles(s)
    out = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = x.float()
        if w is not None:
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        out.append(_turn(y, cos, sin, s["case"]["interleaved"]).to(x.dtype))
    return tuple(out)


def _plain_rotary_grad(s):
    cos, sin = _angles(s)
    dx, dw = [], []
    for dy, x, w in ((s["dq"], s["q"], s["q_weight"]), (s["dk"], s["k"], s["k_weight"])):
        g = _turn(dy.float(), cos, -sin, s["case"]["interleaved"])
        if w is not None:
            n = x.float()
            r = 1 / torch.sqrt(n.square().mean(-1, keepdim=True) + 1e-6)
            n = n * r
            dw.append((g * n).sum((0, 1, 2)).to(w.dtype))
            g = g * w.float()
            g = r * (g - n * (g * n).mean(-1, keepdim=True))
        dx.append(g.to(x.dtype))
    return tuple(dx + dw)


def _slots(s, tokens, count=None):
    """Where tokens 0 .. of each sequence stand, from its start on: (page, slot, whether there is one), [batch, tokens] each."""
    page = s["case"]["page"]
    at = s["start"].long()[:, None] + torch.arange(tokens, device=s["table"].device)[None, :]
    there = torch.ones_like(at, dtype=torch.bool) if count is None else at < (s["start"] + count)[:, None]
    pid = s["table"].long().gather(1, (at // page).clamp(max=s["table"].shape[1] - 1))
    return pid.clamp(min=0), at % page, there


def _plain_append(s):
    b, t = s["k"].shape[:2]
    pid, slot, _ = _slots(s, t)
    for name in ("k", "v"):
        code, e = _to_4bit(s[name].float())
        packed = _to_bytes(code)
        if name == "k":
            s["k_cache"][pid, :, slot] = packed
        else:
            s["v_cache"][pid, :, slot // 4, :, slot % 4] = packed.reshape(b, t, packed.shape[2], -1, 4)
        s[name + "_scales"].view(torch.uint8)[pid, :, :, slot] = e
    return _values_at(s, pid, slot)


def _numbers(packed, scales):
    """The numbers of packed codes [.., dim / 2] with scale bytes [.., ceil(dim / 32)], in 32 bits."""
    code = torch.stack([packed & 15, packed >> 4], -1).flatten(-2).to(torch.int32)
    size = code & 7
    # A code's two exponent bits and one mantissa bit: 0 and 0.5, then (1 or 1.5) * 2^(exponent - 1).
    v = torch.where(size < 2, size.float() * 0.5, (1 + (size & 1).float() * 0.5) * _power(126 + (size >> 1)))
    v = torch.where(code > 7, -v, v)
    power = torch.where(scales == NAN, math.nan, _power(scales.to(torch.int32).clamp(1, 254)))
    return v * power.repeat_interleave(BLOCK, -1)[..., :v.shape[-1]]


def _values_at(s, pid, slot):
    k = _numbers(s["k_cache"][pid, :, slot], s["k_scales"].view(torch.uint8)[pid, :, :, slot])
    v = _numbers(s["v_cache"][pid, :, slot // 4, :, slot % 4].flatten(-2), s["v_scales"].view(torch.uint8)[pid, :, :, slot])
    dtype = TYPES[s["case"]["type"]]
    return k.to(dtype), v.to(dtype)


def _plain_read(s):
    pid, slot, there = _slots(s, s["case"]["longest"], s["count"])
    k, v = _values_at(s, pid, slot)
    there = there[..., None, None]
    return torch.where(there, k, 0.0), torch.where(there, v, 0.0)


def _plain_attention(s):
    case = s["case"]
    b, t, hq, dim = s["q"].shape
    heads, group, page = case["heads"], case["group"], case["page"]
    pid = s["table"].long().clamp(min=0)
    keys = _numbers(s["k_cache"][pid], s["k_scales"].view(torch.uint8)[pid].transpose(3, 4))      # [b, column, h, page, d]
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
    values = s["v_cache"][pid].transpose(4, 5).flatten(5).flatten(3, 4)                           # [b, column, h, page, d / 2]
    values = _numbers(values, s["v_scales"].view(torch.uint8)[pid].transpose(3, 4))
    values = values.permute(0, 2, 1, 3, 4).reshape(b, heads, -1, dim)
    o = (w.reshape(b, heads, t * group, -1) @ values).reshape(b, heads, t, group, dim)
    o = torch.where(total > 0, o / total, 0.0)
    return o.permute(0, 2, 1, 3, 4).reshape(b, t, hq, dim).to(s["q"].dtype)


_PLAIN = {"rotary": _plain_rotary, "rotary_grad": _plain_rotary_grad, "append": _plain_append, "read": _plain_read,
          "attention": _plain_attention}


def _own_rotary(s):
    from paper_1905_13298_amd import ops
    return ops.rotary_norm(s["q"], s["k"], s["positions"], s["frequencies"], s["q_weight"], s["k_weight"], sections=s["sections"],
                           interleaved=s["case"]["interleaved"], eps=1e-6)


def _own_rotary_grad(s):
    from paper_1905_13298_amd import ops
    got = ops.rotary_norm_backward(s["dq"], s["dk"], s["q"], s["k"], s["positions"], s["frequencies"], s["q_weight"], s["k_weight"],
                                   sections=s["sections"], interleaved=s["case"]["interleaved"], eps=1e-6)
    return tuple(g for g in got if g is not None)


def _held(s):
    return s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"]


def _own_append(s):
    from paper_1905_13298_amd import ops
    ops.kv_cache_fp4_append(s["k"], s["v"], *_held(s), s["table"], s["start"])
    return ops.kv_cache_fp4_read(*_held(s), s["table"], s["start"], s["case"]["tokens"], dtype=TYPES[s["case"]["type"]])


def _own_read(s):
    from paper_1905_13298_amd import ops
    return ops.kv_cache_fp4_read(*_held(s), s["table"], s["start"], s["case"]["longest"], s["count"], dtype=TYPES[s["case"]["type"]])


def _own_attention(s):
    from paper_1905_13298_amd import ops
    return ops.attention_fp4(s["q"], *_held(s), s["table"], s["length"], count=s["count"], window=s["case"]["window"])


_OWN = {"rotary": _own_rotary, "rotary_grad": _own_rotary_grad, "append": _own_append, "read": _own_read,
        "attention": _own_attention}


# ---------------------------------------------------------------------------
# What a pass cannot do without.


def _lengths(case):
    """The expected sum of the lengths of a case's sequences."""
    b, longest = case["batch"], case["longest"]
    if case["kind"] == "read":
        return longest + (b - 1) * longest * 7 / 8
    low = longest * 7 / 8 if case["even"] else 0 if b > 3 else max(1, longest // 2)
    rest = (low + longest) / 2 if not case["even"] or b <= 3 else low + longest / 128
    return longest + (b - 1) * rest


def work(case):
    kind, e = case["kind"], {"bf16": 2, "f16": 2, "f32": 4}[case["type"]]
    if kind in ("rotary", "rotary_grad"):
        tokens = case["batch"] * case["tokens"]
        n = tokens * (case["heads"] + case["kv_heads"]) * case["dim"]
        small = 4 * tokens * case["axes"] + 8 * case["pairs"] + 2 * case["dim"] * e * case["norm"]
        if kind == "rotary":
            return {"bytes": 2 * n * e + small, "flops": n * (7 if case["norm"] else 3)}
        return {"bytes": (3 if case["norm"] else 2) * n * e + small, "flops": n * (16 if case["norm"] else 3)}
    held = case["dim"] / 2 + (case["dim"] + BLOCK - 1) // BLOCK              # of a token's head
    if kind == "append":
        n = 2 * case["batch"] * case["tokens"] * case["heads"]
        return {"bytes": 2 * n * (case["dim"] * e + held), "flops": 4 * n * case["dim"]}
    if kind == "read":
        out = 2 * case["batch"] * case["longest"] * case["heads"] * case["dim"]
        return {"bytes": 2 * _lengths(case) * case["heads"] * held + out * e, "flops": out}
    total, rows = _lengths(case), case["batch"] * case["tokens"] * case["heads"] * case["group"]
    mean = total / case["batch"]
    seen = max(1.0, mean - (min(mean, case["tokens"]) - 1) / 2)
    kept = mean
    if case["window"]:
        seen, kept = min(seen, case["window"]), min(mean, case["window"] + case["tokens"])
    return {"bytes": 2 * case["batch"] * kept * case["heads"] * held + 2 * rows * case["dim"] * e,
            "flops": 4 * rows * seen * case["dim"]}


# ---------------------------------------------------------------------------
# The definitions in 64 bits, one head, token or page at a time.


def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed))


def _exact_partners(case, device):
    """For each element of a head its pair's other element, the angle's sign in its sine's term, and its pair (-1: none)."""
    dim, pairs = case["dim"], case["pairs"]
    other, sign, pair = list(range(dim)), [0.0] * dim, [-1] * dim
    for i in range(pairs):
        first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + pairs)
        other[first], other[second], sign[first], sign[second], pair[first], pair[second] = second, first, -1.0, 1.0, i, i
    return torch.tensor(other, device=device), torch.tensor(sign, dtype=torch.float64, device=device), pair


def _exact_angles(case, s, pair):
    """[batch, tokens, dim]."""
    sections = s["sections"] or (case["pairs"],)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    positions = s["positions"] if s["sections"] else s["positions"][None]
    angle = torch.zeros(*positions.shape[1:], case["dim"], dtype=torch.float64, device=positions.device)
    for d, i in enumerate(pair):
        if i >= 0:
            angle[:, :, d] = positions[axis[i]].double() * s["frequencies"][i]
    return angle


def _exact_rotary(case, s):
    other, sign, pair = _exact_partners(case, s["q"].device)
    angle = _exact_angles(case, s, pair)
    got = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = torch.empty(x.shape, dtype=torch.float64, device=x.device)
        for h in range(x.shape[2]):
            v = x[:, :, h].double()
            if w is not None:
                v = v * torch.pow(torch.sum(v * v, 2, keepdim=True) / case["dim"] + 1e-6, -0.5) * w.double()
            y[:, :, h] = v * torch.cos(angle) + sign * v[:, :, other] * torch.sin(angle)
        got.append(y)
    return tuple(got)


def _exact_rotary_grad(case, s):
    other, sign, pair = _exact_partners(case, s["q"].device)
    angle = _exact_angles(case, s, pair)
    dx, dw = [], []
    for dy, x, w in ((s["dq"], s["q"], s["q_weight"]), (s["dk"], s["k"], s["k_weight"])):
        got = torch.empty(x.shape, dtype=torch.float64, device=x.device)
        sums = torch.zeros(case["dim"], dtype=torch.float64, device=x.device)
        for h in range(x.shape[2]):
            # An element reaches its own result with the cosine and its partner's with that one's sine.
            u = dy[:, :, h].double()
            g = u * torch.cos(angle) + (u * sign * torch.sin(angle))[:, :, other]
            if w is not None:
                v = x[:, :, h].double()
                r = torch.pow(torch.sum(v * v, 2, keepdim=True) / case["dim"] + 1e-6, -0.5)
                sums += torch.sum(g * v * r, (0, 1))
                inner = torch.sum(g * w.double() * v, 2, keepdim=True)
                g = g * w.double() * r - v * (r.pow(3) * inner / case["dim"])
            got[:, :, h] = g
        dx.append(got)
        if w is not None:
            dw.append(sums)
    return tuple(dx + dw)


_SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_held(x):
    """x [.., dim] as a 4-bit cache holds it: the nearest number of each, at a tie the one with the even code."""
    out = x.double()
    for c in range(0, x.shape[-1], 32):
        part = out[..., c:c + 32]
        fine = torch.isfinite(part).all(-1, keepdim=True)
        part = torch.where(fine, part, 0.0)
        largest = part.abs().amax(-1, keepdim=True)
        scale = torch.exp2(torch.ceil(torch.log2(largest.clamp(min=1e-300) / 6.0))).clamp(2.0 ** -23, 2.0 ** 13)
        y = part.abs() / scale
        best, off = torch.zeros_like(y), y.clone()
        for i in range(1, 8):
            away = (y - _SIZES[i]).abs()
            better = (away < off) | ((away == off) & (i % 2 == 0))
            best, off = torch.where(better, _SIZES[i], best), torch.where(better, away, off)
        out[..., c:c + 32] = torch.where(fine, torch.sign(part) * best * scale, math.nan)
    return out


def _exact_append(case, s):
    return _exact_held(s["k"]), _exact_held(s["v"])


def _exact_pages(s, case, i, n, h):
    """Keys and values [n, dim] of the first n tokens of sequence i's head h."""
    page, dim = case["page"], case["dim"]
    rows = s["table"][i, :(n - 1) // page + 1].long()
    names = torch.tensor([*_SIZES, *(-v for v in _SIZES)], dtype=torch.float64, device=rows.device)
    k, v = s["k_cache"][rows, h].reshape(-1, dim // 2)[:n].long(), s["v_cache"][rows, h].long()
    v = torch.cat([v[:, :, :, j].flatten(2)[:, :, None] for j in range(4)], 2).reshape(-1, dim // 2)[:n]
    got = []
    for b, scales in ((k, s["k_scales"]), (v, s["v_scales"])):
        x = torch.empty(n, dim, dtype=torch.float64, device=rows.device)
        x[:, 0::2], x[:, 1::2] = names[b % 16], names[b // 16]
        by_token = scales[rows, h].double()                      # [page, block, slot]
        for c in range(by_token.shape[1]):
            x[:, 32 * c:32 * c + 32] *= by_token[:, c].reshape(-1)[:n, None]
        got.append(x)
    return got


def _exact_read(case, s):
    b, longest, heads, dim = case["batch"], case["longest"], case["heads"], case["dim"]
    k = torch.zeros(b, longest, heads, dim, dtype=torch.float64, device=s["table"].device)
    v = torch.zeros_like(k)
    for i, n in enumerate(s["count"].cpu().tolist()):
        for h in range(heads if n else 0):
            k[i, :n, h], v[i, :n, h] = _exact_pages(s, case, i, n, h)
    return k, v


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
        own_place = torch.arange(n - c, n, device=out.device)[:, None]
        other = torch.arange(n, device=out.device)[None, :]
        hidden = other > own_place
        if case["window"]:
            hidden |= other <= own_place - case["window"]
        for h in range(case["heads"]):
            k, v = _exact_pages(s, case, i, n, h)
            k = k.t().contiguous()
            for g in range(case["group"]):
                q = s["q"][i, :c, h * case["group"] + g].double()
                p = torch.softmax(torch.mm(q, k).mul_(dim ** -0.5).masked_fill_(hidden, -math.inf), 1)
                out[i, :c, h * case["group"] + g] = torch.mm(p, v)
    return out


_EXACT = {"rotary": _exact_rotary, "rotary_grad": _exact_rotary_grad, "append": _exact_append, "read": _exact_read,
          "attention": _exact_attention}
