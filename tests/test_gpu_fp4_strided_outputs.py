"""Outputs with strides of their own, as the C interface takes them: what the wrappers' packed outputs hold, and the gaps as they were."""
import ctypes
import math

import pytest
import torch

from paper_1905_13298_amd import _native, ops

from .test_gpu_fp4 import BF16, DEV, F16, F32, filled_cache, normal

pytestmark = pytest.mark.gpu

TYPE = {F32: 0, F16: 1, BF16: 2}
MARK = 77.0


class Spaced:
    """An output [batch, tokens, heads, dim] of which vectors begin anywhere: sequence, token and head strides with gaps."""

    def __init__(self, shape, dtype, gap):
        b, t, h, d = shape
        head = d + gap
        token = h * head + 5
        self.strides = (t * token + 3, token, head)
        self.flat = torch.full((1 + b * self.strides[0],), MARK, dtype=dtype, device=DEV)
        self.view = self.flat[1:].as_strided(shape, (*self.strides, 1), 1)
        self.c = (ctypes.c_int64 * 3)(*self.strides)

    def ptr(self):
        return self.view.data_ptr()

    def holds(self, want):
        assert torch.equal(self.view, want)
        self.view.fill_(MARK)
        assert torch.all(self.flat == MARK)


def strides(t):
    return (ctypes.c_int64 * 3)(*t.stride()[:3])


def call(name, *args):
    torch.cuda.synchronize()
    _native.call(name, *args, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dim,pairs,interleaved", [(64, 32, 0), (40, 12, 0), (34, 9, 1), (128, 64, 1)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gap", [1, 8])
def test_rotation_and_gradient(dim, pairs, interleaved, dtype, gap):
    batch, tokens, heads, kv = 2, 5, 9, 3
    q, k = normal(1, batch, tokens, heads, dim).to(DEV, dtype), normal(2, batch, tokens, kv, dim).to(DEV, dtype)
    at = torch.arange(batch * tokens, dtype=torch.int32, device=DEV).reshape(batch, tokens)
    f, w = ops.rotary_frequencies(pairs), (1 + normal(3, dim, std=0.2)).to(DEV, dtype)
    sizes, sp, t = (batch, tokens, heads, kv, dim, pairs, 1), (ctypes.c_int64 * 3)(0, tokens, 1), TYPE[dtype]
    qo, ko = Spaced(q.shape, dtype, gap), Spaced(k.shape, dtype, gap)
    call("ds_rotary_norm", q.data_ptr(), k.data_ptr(), at.data_ptr(), f.data_ptr(), w.data_ptr(), w.data_ptr(), qo.ptr(), ko.ptr(), *sizes, None,
         strides(q), strides(k), sp, qo.c, ko.c, interleaved, 1e-6, t, t, 5)
    want = ops.rotary_norm(q, k, at, f, w, w, interleaved=bool(interleaved))
    qo.holds(want[0])
    ko.holds(want[1])
    dq, dk, dqw, dkw = Spaced(q.shape, dtype, gap), Spaced(k.shape, dtype, gap), torch.empty_like(w), torch.empty_like(w)
    size = _native.lib().ds_rotary_norm_backward_scratch_bytes(batch, tokens, heads, kv, dim)
    scratch = torch.empty(size, dtype=torch.uint8, device=DEV)
    call("ds_rotary_norm_backward", want[0].data_ptr(), want[1].data_ptr(), q.data_ptr(), k.data_ptr(), at.data_ptr(), f.data_ptr(), w.data_ptr(),
         w.data_ptr(), dq.ptr(), dk.ptr(), dqw.data_ptr(), dkw.data_ptr(), *sizes, None, strides(q), strides(k), strides(q), strides(k), sp, dq.c, dk.c,
         interleaved, 1e-6, t, t, 5, scratch.data_ptr(), size)
    grads = ops.rotary_norm_backward(*want, q, k, at, f, w, w, interleaved=bool(interleaved))
    dq.holds(grads[0])
    dk.holds(grads[1])
    assert torch.equal(dqw, grads[2]) and torch.equal(dkw, grads[3])


@pytest.mark.parametrize("tokens,dim,dtype", [(3, 80, BF16), (40, 48, F32), (1500, 128, F16)])       # (one token a thread, and four)
def test_read(tokens, dim, dtype):
    heads, page, batch = 3, 32, 2
    columns = tokens // page + 2
    cache = filled_cache(ops, batch * columns, heads, page, dim)
    table = torch.arange(batch * columns, dtype=torch.int32, device=DEV).reshape(batch, columns)
    start, count = torch.tensor([0, 13], dtype=torch.int32, device=DEV), torch.tensor([tokens, tokens - 1], dtype=torch.int32, device=DEV)
    want = ops.kv_cache_fp4_read(*cache, table, start, tokens, count, dtype=dtype)
    k, v = Spaced(want[0].shape, dtype, 3), Spaced(want[0].shape, dtype, 1)
    call("ds_kv_cache_fp4_read", *(c.data_ptr() for c in cache), table.data_ptr(), start.data_ptr(), count.data_ptr(), k.ptr(), v.ptr(), batch, tokens,
         heads, dim, page, batch * columns, columns, columns, k.c, v.c, TYPE[dtype])
    k.holds(want[0])
    v.holds(want[1])


@pytest.mark.parametrize("tokens,group,length", [(1, 4, 300), (1, 4, 9000), (9, 3, 300), (70, 2, 300)])
@pytest.mark.parametrize("dim,dtype", [(48, F16), (128, BF16), (208, BF16)])
def test_attention(tokens, group, length, dim, dtype):
    heads, page, batch = 2, 32, 2
    columns = (length + page - 1) // page
    cache = filled_cache(ops, batch * columns, heads, page, dim)
    table = torch.arange(batch * columns, dtype=torch.int32, device=DEV).reshape(batch, columns)
    lengths = torch.tensor([length, length // 3], dtype=torch.int32, device=DEV)
    q = normal(4, batch, tokens, heads * group, dim).to(DEV, dtype)
    want = ops.attention_fp4(q, *cache, table, lengths)
    o = Spaced(q.shape, dtype, 3)
    size = _native.lib().ds_attention_fp4_scratch_bytes(batch, tokens, heads, group, dim, page, columns)
    scratch = torch.empty(max(size, 1), dtype=torch.uint8, device=DEV)
    call("ds_attention_fp4", q.data_ptr(), *(c.data_ptr() for c in cache), table.data_ptr(), lengths.data_ptr(), None, o.ptr(), batch, tokens, heads, group,
         dim, page, batch * columns, columns, columns, strides(q), o.c, 1 / math.sqrt(dim), 0, TYPE[dtype], scratch.data_ptr() if size else None, size)
    o.holds(want)
