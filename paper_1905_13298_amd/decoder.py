"""A decoder of a language model on the 8-bit operators: prompts and single tokens over a paged cache.

One layer is ten calls: RMS norm (with the residual's sum, 8-bit output), the product that
forms queries, keys and values, the append to the cache, attention over it, the attention's output
in 8 bits, its product, the second norm, the gate and value product, silu(gate) * value in 8 bits
and the last product. Between the operators only 8-bit rows with their scales and 16-bit results
pass through memory. Weights are shift codes (sign and power of two, exact in 8 bits) or
float matrices, which are rounded once here. Positions enter through x alone: what rotates
queries and keys is not part of the layer.
"""
from __future__ import annotations

import torch

from . import ops


def weights(w, cols: int, code_bits: int = 5):
    """(w8, scales) of packed shift codes [rows, words] (int32) or a float matrix [rows, cols]."""
    if w.dtype == torch.int32:
        return ops.shift_weights_to_fp8(w, cols, code_bits)
    if w.dim() != 2 or w.shape[1] != cols:
        raise ValueError(f"a weight matrix must have {cols} columns, got {tuple(w.shape)}")
    return ops.quantize_weights_fp8(w)


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


class DecoderLayer:
    """params: "norm1", "norm2" [hidden]; "qkv" [(heads + 2 kv_heads) dim, hidden], "out" [hidden, heads dim],
    "gate_up" [2 inner, hidden] (the gates' rows first), "down" [hidden, inner], as `weights` takes them."""

    def __init__(self, params, heads: int, kv_heads: int, dim: int, inner: int, code_bits: int = 5, window: int = 0):
        if heads <= 0 or kv_heads <= 0 or heads % kv_heads:
            raise ValueError(f"{heads} query heads over {kv_heads} heads")
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

    def __call__(self, x, residual, cache, table, start, length, count=None):
        """x [batch, tokens, hidden] and the residual (None before the first layer) -> the same two for the
        next layer; the layer's output is their sum. The tokens are appended at `start` (length = start + count)."""
        batch, tokens, hidden = x.shape
        qkv, h, _ = self.qkv(x.reshape(-1, hidden), None if residual is None else residual.reshape(-1, hidden))
        heads = [self.heads, self.kv_heads, self.kv_heads]
        q, k, v = qkv.view(batch, tokens, sum(heads), self.dim).split(heads, dim=2)
        ops.kv_cache_append(k, v, *cache, table, start, count)
        o = ops.attention_fp8(q, *cache, table, length, count, window=self.window)
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
        self.caches = [ops.kv_cache(batch * columns, layer.kv_heads, page, layer.dim, dev) for layer in layers]

    def reset(self):
        """Forgets every sequence. (A page written from its first token on starts afresh.)"""
        self.length.zero_()

    def __call__(self, x, count=None):
        """x [batch, tokens, hidden] of the next tokens, the first count[b] of them (all without count) those
        of sequence b (all where it is more) -> the last norm's output. A prompt and single tokens alike; with one
        shape a call it can be captured into a graph. Tokens past the capacity are not kept: they count in `length`,
        come out as tokens that see what was kept, and are seen by none."""
        self._check(x, count)
        length = self.length + (x.shape[1] if count is None else count.clamp(0, x.shape[1]))
        residual = None
        for layer, cache in zip(self.layers, self.caches):
            x, residual = layer(x, residual, cache, self.table, self.length, length, count)
        hidden = x.shape[2]
        y, _, _, _ = ops.rms_norm(x.reshape(-1, hidden), self.norm, residual.reshape(-1, hidden), quantize=False)
        self.length.copy_(length)      # (once nothing can be refused any more)
        return y.view(x.shape)

    def _check(self, x, count):
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
        ops._same_device(x.device, count, self.length, *norms)
