"""A decoder of a language model on the 8-bit operators: prompts and single tokens over a paged cache.

One layer is ten calls: RMS norm (with the residual's sum, 8-bit output), the product that
forms queries, keys and values, the append to the cache, attention over it, the attention's output
in 8 bits, its product, the second norm, the gate and value product, silu(gate) * value in 8 bits
and the last product; with a `Rotary`, which norms queries and keys and turns them by their positions
in front of the append, eleven (without one positions enter through x alone). Between the
operators only 8-bit rows with their scales and 16-bit results pass through memory. The cache holds
8 bits an element or 4. Weights are shift codes (sign and power of two, exact in 8 bits) or float
matrices, which are rounded once here.
"""
from __future__ import annotations

import operator

import torch

from . import ops


def weights(w, cols: int, code_bits: int = 5):
    """(w8, scales) of packed shift codes [rows, words] (int32) or a float matrix [rows, cols]."""
    if w.dtype == torch.int32:
        return ops.shift_weights_to_fp8(w, cols, code_bits)
    if w.dim() != 2 or w.shape[1] != cols:
        raise ValueError(f"a weight matrix must have {cols} columns, got {tuple(w.shape)}")
    return ops.quantize_weights_fp8(w)


# What makes, fills and reads a cache of so many bits an element.
_CACHES = {8: (ops.kv_cache, ops.kv_cache_append, ops.attention_fp8),
           4: (ops.kv_cache_fp4, ops.kv_cache_fp4_append, ops.attention_fp4)}


class NormLinear:
    """y = rms_norm(x + residual) w^T, the normalised rows in 8 bits."""

    def __init__(self, norm, w8, scales, eps: float = 1e-6):
        self.norm, self.w8, self.scales, self.eps = norm, w8, scales, eps

    def __call__(self, x, residual=None):
        """(y, h, rstd): h = x + residual goes on as the residual, h and rstd to `backward`."""
        n8, scales, h, rstd = ops.rms_norm(x, self.norm, residual, self.eps)
        return ops.linear_fp8(n8, scales, self.w8, self.scales, out_dtype=x.dtype), h, rstd

    def backward(self, dy, h, rstd, dh=None):
        """(gradient of x and of the residual, gradient of the norm's weight)."""
        dn = ops.linear_fp8_backward_data(*ops.quantize_fp8(dy), self.w8, self.scales, out_dtype=h.dtype)
        return ops.rms_norm_backward(dn, h, self.norm, rstd, dh)


class Rotary:
    """Query and key heads turned by their positions, normed before where there are weights [dim] (of the
    activations' type or float32): `ops.rotary_norm` with what of it a model keeps."""

    def __init__(self, frequencies, q_norm=None, k_norm=None, sections=None, interleaved: bool = False, eps: float = 1e-6):
        self.frequencies, self.q_norm, self.k_norm = frequencies, q_norm, k_norm
        self.sections = None if sections is None else tuple(operator.index(n) for n in sections)
        self.interleaved, self.eps = interleaved, eps

    @property
    def axes(self) -> int:
        return 1 if self.sections is None else len(self.sections)

    def check(self, x, dim: int, positions):
        """Refuses activations x [batch, tokens, hidden] of heads of `dim`, or positions (None: not given), that a call would refuse."""
        if positions is not None and positions.shape != x.shape[:2] and positions.shape != (self.axes, *x.shape[:2]):
            raise ValueError(f"positions must be [{x.shape[0]}, {x.shape[1]}] or [{self.axes}, {x.shape[0]}, {x.shape[1]}], got {tuple(positions.shape)}")
        pairs = self.frequencies.numel()
        ops._vector(self.frequencies, "frequencies", (torch.float32, torch.float64), pairs)
        if dim % 2 or not 0 < pairs <= dim // 2:
            raise ValueError(f"{pairs} pairs of heads of {dim}")
        if self.sections is not None and (sum(self.sections) != pairs or min(self.sections) < 0 or len(self.sections) > 4):
            raise ValueError(f"sections {self.sections} of {pairs} pairs")
        if not self.eps >= 0:
            raise ValueError(f"eps must be >= 0, got {self.eps}")
        for norm in (self.q_norm, self.k_norm):
            if norm is not None:
                ops._vector(norm, "a head's norm", (x.dtype, torch.float32), dim)
        if self.q_norm is not None and self.k_norm is not None and self.q_norm.dtype != self.k_norm.dtype:
            raise TypeError(f"the norms of queries and keys are {self.q_norm.dtype} and {self.k_norm.dtype}")
        ops._same_device(x.device, self.frequencies, self.q_norm, self.k_norm)

    def __call__(self, q, k, positions):
        """(q', k') of q and k [batch, tokens, heads, dim]; positions as `ops.rotary_norm` takes them."""
        return ops.rotary_norm(q, k, positions, self.frequencies, self.q_norm, self.k_norm, self.sections, self.interleaved, self.eps)

    def backward(self, dq, dk, q, k, positions):
        """Gradients of q, of k and of the two norms' weights (None without them) from those of the results."""
        return ops.rotary_norm_backward(dq, dk, q, k, positions, self.frequencies, self.q_norm, self.k_norm, self.sections, self.interleaved,
                                        self.eps)


class DecoderLayer:
    """params: "norm1", "norm2" [hidden]; "qkv" [(heads + 2 kv_heads) dim, hidden], "out" [hidden, heads dim],
    "gate_up" [2 inner, hidden] (the gates' rows first), "down" [hidden, inner], as `weights` takes them.
    rotary: a Rotary for queries and keys, or None; cache_bits: 8 or 4, what the layer's cache holds an element in."""

    def __init__(self, params, heads: int, kv_heads: int, dim: int, inner: int, code_bits: int = 5, window: int = 0,
                 rotary: Rotary | None = None, cache_bits: int = 8):
        if heads <= 0 or kv_heads <= 0 or heads % kv_heads:
            raise ValueError(f"{heads} query heads over {kv_heads} heads")
        if cache_bits not in _CACHES:
            raise ValueError(f"a cache holds 8 or 4 bits an element, not {cache_bits}")
        if not 0 <= operator.index(window) < 2 ** 31:
            raise ValueError(f"window must be in [0, 2^31), got {window}")
        self.rotary, self.cache_bits = rotary, cache_bits
        hidden = params["norm1"].shape[0]
        self.heads, self.kv_heads, self.dim, self.window = heads, kv_heads, dim, window
        rows = {"qkv": (heads + 2 * kv_heads) * dim, "out": hidden, "gate_up": 2 * inner, "down": hidden}
        cols = {"qkv": hidden, "out": heads * dim, "gate_up": hidden, "down": inner}
        for name, n in rows.items():
            if params[name].shape[0] != n:
                raise ValueError(f"{name} must have {n} rows, got {params[name].shape[0]}")
        w = {name: weights(params[name], cols[name], code_bits) for name in rows}
        self.qkv = NormLinear(params["norm1"], *w["qkv"])
        self.gate_up = NormLinear(params["norm2"], *w["gate_up"])
        self.out, self.down = w["out"], w["down"]

    def cache(self, pages: int, page: int, device):
        """An empty cache for the layer."""
        return _CACHES[self.cache_bits][0](pages, self.kv_heads, page, self.dim, device)

    def __call__(self, x, residual, cache, table, start, length, count=None, positions=None):
        """x [batch, tokens, hidden] and the residual (None before the first layer) -> the same two for the
        next layer; the layer's output is their sum. The tokens are appended at `start` (length = start + count);
        positions: what the layer's rotary goes by."""
        batch, tokens, hidden = x.shape
        qkv, h, _ = self.qkv(x.reshape(-1, hidden), None if residual is None else residual.reshape(-1, hidden))
        heads = [self.heads, self.kv_heads, self.kv_heads]
        q, k, v = qkv.view(batch, tokens, sum(heads), self.dim).split(heads, dim=2)
        if self.rotary is not None:
            q, k = self.rotary(q, k, positions)
        _, append, attention = _CACHES[self.cache_bits]
        append(k, v, *cache, table, start, count)
        o = attention(q, *cache, table, length, count, window=self.window)
        a = ops.linear_fp8(*ops.quantize_fp8(o.view(batch * tokens, self.heads * self.dim)), *self.out, out_dtype=x.dtype)
        gu, h, _ = self.gate_up(a, h)
        gate, up = gu.chunk(2, dim=1)
        y = ops.linear_fp8(*ops.quantize_fp8(up, gate), *self.down, out_dtype=x.dtype)
        return y.view(x.shape), h.view(x.shape)


class Decoder:
    """Layers, their caches and the sequences' lengths. Sequence b owns the pages b * columns ..
    of every layer's cache; `length` [batch] (int32, on the device) counts its tokens."""

    def __init__(self, layers, norm, batch: int, tokens: int, page: int = 64):
        self.layers, self.norm = layers, norm
        dev = norm.device
        columns = (tokens + page - 1) // page
        self.capacity = columns * page
        self.table = torch.arange(batch * columns, dtype=torch.int32, device=dev).view(batch, columns)
        self.length = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.caches = [layer.cache(batch * columns, page, dev) for layer in layers]

    def reset(self):
        """Forgets every sequence. (A page written from its first token on starts afresh.)"""
        self.length.zero_()

    def __call__(self, x, count=None, positions=None):
        """x [batch, tokens, hidden] of the next tokens, the first count[b] of them (all without count) those
        of sequence b (all where it is more) -> the last norm's output. A prompt and single tokens alike; with one
        shape a call it can be captured into a graph. Tokens past the capacity are not kept: they count in `length`,
        come out as tokens that see what was kept, and are seen by none. positions (int32 [batch, tokens], or [axes, batch,
        tokens]): what the layers' rotaries go by; without them a token's place in its sequence, on every axis."""
        self._check(x, count, positions)
        length = self.length + (x.shape[1] if count is None else count.clamp(0, x.shape[1]))
        at = self._positions(x.shape[1], positions)
        residual = None
        for layer, cache in zip(self.layers, self.caches):
            turned = () if layer.rotary is None else (at[layer.rotary.axes],)
            x, residual = layer(x, residual, cache, self.table, self.length, length, count, *turned)
        hidden = x.shape[2]
        y, _, _, _ = ops.rms_norm(x.reshape(-1, hidden), self.norm, residual.reshape(-1, hidden), quantize=False)
        self.length.copy_(length)      # (once nothing can be refused any more)
        return y.view(x.shape)

    def _positions(self, tokens: int, positions):
        """The positions for each number of axes that a layer's rotary has."""
        axes = {layer.rotary.axes for layer in self.layers if layer.rotary is not None}
        if axes and positions is None:
            positions = self.length[:, None] + torch.arange(tokens, dtype=torch.int32, device=self.length.device)
        return {n: positions if n == 1 or positions.dim() == 3 else positions.expand(n, *positions.shape) for n in axes}

    def _check(self, x, count, positions):
        """Refuses a call before any cache is written: a decoder is as it was behind an error."""
        ops._dev_as(x, "x", (torch.bfloat16, torch.float16))
        batch, hidden = self.length.shape[0], self.norm.shape[0]
        if x.dim() != 3 or x.shape[0] != batch or x.shape[2] != hidden:
            raise ValueError(f"x must be [{batch}, tokens, {hidden}], got {tuple(x.shape)}")
        norms = [self.norm] + [n.norm for layer in self.layers for n in (layer.qkv, layer.gate_up)]
        for norm in norms:
            if norm.dtype not in (x.dtype, torch.float32):
                raise TypeError(f"x is {x.dtype}, a norm's weight {norm.dtype}")
        if count is not None:
            ops._vector(count, "count", (torch.int32,), batch)
        ops._same_device(x.device, count, positions, self.length, *norms)
        rotaries = [layer.rotary for layer in self.layers if layer.rotary is not None]
        if positions is not None:
            if not rotaries:
                raise ValueError("positions without a layer that goes by them")
            ops._dev_as(positions, "positions", (torch.int32,))
        for layer in self.layers:
            if layer.rotary is not None:
                layer.rotary.check(x, layer.dim, positions)
