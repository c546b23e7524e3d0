"""Argument checks of the rotation and of the 4-bit cache's operators that need no GPU: they run before
any device access, so bad sizes, types, strides and pointers are refused with the documented status."""
import ctypes

import pytest
import torch

from paper_1905_13298_amd import _native, ops

OK, NULLP, SHAPE, ARG, SMALL, CODE, HIP, UNSUP = range(8)
P = [0x100000 * (i + 1) for i in range(14)]       # never dereferenced
F32, F16, BF16, E4M3, E5M2, F64 = range(6)
KEPT = []


def strides(*v):
    KEPT.append((ctypes.c_int64 * 3)(*v))
    return ctypes.cast(KEPT[-1], ctypes.c_void_p)


def sections(*v):
    KEPT.append((ctypes.c_int32 * len(v))(*v))
    return ctypes.cast(KEPT[-1], ctypes.c_void_p)


ST, PS = strides(1024, 128, 64), strides(64, 8, 1)


def status(name, *args):
    return getattr(_native.lib(), name)(*args)


def rotary(q=P[0], k=P[1], pos=P[2], f=P[3], qw=P[4], kw=P[5], qo=P[6], ko=P[7], batch=1, tokens=2, heads=2, kv=2, dim=64, pairs=32, axes=1,
           sec=None, sq=ST, sk=ST, sp=PS, so=ST, sko=ST, inter=0, eps=1e-6, t=BF16, wt=BF16, ft=F64):
    return status("ds_rotary_norm", q, k, pos, f, qw, kw, qo, ko, batch, tokens, heads, kv, dim, pairs, axes, sec, sq, sk, sp, so, sko, inter,
                  eps, t, wt, ft, None)


def rotary_grad(dqo=P[0], dko=P[1], q=P[2], k=P[3], pos=P[4], f=P[5], qw=P[6], kw=P[7], dq=P[8], dk=P[9], dqw=P[10], dkw=P[11], batch=1, tokens=2,
                heads=2, kv=2, dim=64, pairs=32, axes=1, sec=None, st=ST, sq=ST, sk=ST, sp=PS, sdq=ST, sdk=ST, inter=0, eps=1e-6, t=BF16, wt=F32,
                ft=F32, scratch=P[12], size=1 << 20):
    return status("ds_rotary_norm_backward", dqo, dko, q, k, pos, f, qw, kw, dq, dk, dqw, dkw, batch, tokens, heads, kv, dim, pairs, axes, sec,
                  st, st, sq, sk, sp, sdq, sdk, inter, eps, t, wt, ft, scratch, size, None)


COMMON = [
    (NULLP, dict(pos=None)), (NULLP, dict(f=None)), (NULLP, dict(k=None)), (NULLP, dict(q=None)), (NULLP, dict(sp=None)), (NULLP, dict(sq=None)),
    (NULLP, dict(sk=None)), (NULLP, dict(axes=2)), (SHAPE, dict(batch=-1)), (SHAPE, dict(tokens=-1)), (SHAPE, dict(heads=0)), (SHAPE, dict(kv=-1)),
    (SHAPE, dict(dim=0)), (SHAPE, dict(pairs=0)), (SHAPE, dict(pairs=33)), (SHAPE, dict(axes=0)), (UNSUP, dict(dim=65)), (UNSUP, dict(dim=258)),
    (UNSUP, dict(axes=5, sec=sections(8, 8, 8, 4, 4))), (UNSUP, dict(heads=65536)), (UNSUP, dict(batch=1 << 16, tokens=1 << 16)),
    (UNSUP, dict(batch=1 << 40, tokens=1 << 40)),
    (ARG, dict(axes=2, sec=sections(16, 15))), (ARG, dict(axes=2, sec=sections(33, -1))), (ARG, dict(axes=2, sec=sections(32, 32))),
    (ARG, dict(t=E4M3)), (ARG, dict(wt=F16)), (ARG, dict(ft=F16)), (ARG, dict(eps=-1.0)), (ARG, dict(eps=float("nan"))),
    (ARG, dict(sq=strides(1, -1, 1))), (ARG, dict(sp=strides(1, 1, -1))), (UNSUP, dict(batch=2, sq=strides(1 << 61, 128, 64))),
    (UNSUP, dict(tokens=2, sp=strides(1, 1, 1 << 60))), (ARG, {}),           # (ARG in the end: not device memory)
]


@pytest.mark.parametrize("want,kw", COMMON + [
    (NULLP, dict(qo=None)), (NULLP, dict(ko=None)), (NULLP, dict(so=None)), (NULLP, dict(sko=None)), (ARG, dict(qo=P[0])), (ARG, dict(ko=P[6])),
    (ARG, dict(ko=P[2])), (ARG, dict(qw=None, kw=None)), (UNSUP, dict(batch=1 << 15, tokens=1 << 15, dim=2, pairs=1, sq=strides(0, 0, 2))),
])
def test_rotary(want, kw):
    assert rotary(**kw) == want


@pytest.mark.parametrize("want,kw", COMMON + [
    (NULLP, dict(dqo=None)), (NULLP, dict(dko=None)), (NULLP, dict(dq=None)), (NULLP, dict(dk=None)), (NULLP, dict(scratch=None)),
    (SMALL, dict(size=1 * 2 * 64 * 4 - 1)), (NULLP, dict(st=None)), (NULLP, dict(sdq=None)), (NULLP, dict(sdk=None)), (ARG, dict(qw=None)),
    (ARG, dict(kw=None)), (ARG, dict(dq=P[0])), (ARG, dict(dqw=P[6])), (ARG, dict(scratch=P[9])), (ARG, dict(qw=None, dqw=None, q=None, sq=None)),
    (ARG, dict(dqw=None, dkw=None, scratch=None, size=0)),
])
def test_rotary_gradient(want, kw):
    assert rotary_grad(**kw) == want


def test_calls_without_tokens_do_nothing():
    none = dict(q=None, k=None, pos=None, f=None, sq=None, sk=None, sp=None)
    assert rotary(batch=0, qo=None, ko=None, so=None, sko=None, **none) == OK and rotary(tokens=0) == OK
    assert rotary_grad(tokens=0, dqw=None, dkw=None, scratch=None, size=0, **none) == OK
    assert append(batch=0, k=None, v=None) == OK and append(tokens=0) == OK
    assert read(batch=0, k=None, v=None) == OK and read(tokens=0) == OK
    assert attention(batch=0, q=None, o=None) == OK and attention(tokens=0) == OK


def test_scratch_sizes():
    lib = _native.lib()
    need = lib.ds_rotary_norm_backward_scratch_bytes
    assert need(0, 4, 2, 2, 64) == 0 and need(1, 4, 2, 2, 1 << 20) == 0 and need(1, 4, 0, 2, 64) == 0
    assert need(1, 4, 2, 2, 64) == 2 * 64 * 4 and need(1, 4, 2, 0, 64) == 64 * 4
    assert lib.ds_attention_fp4_scratch_bytes(0, 1, 1, 1, 64, 16, 4) == 0
    assert lib.ds_attention_fp4_scratch_bytes(1, 1, 8, 4, 128, 64, 4096) > 0


def append(k=P[0], v=P[1], kc=P[2], vc=P[3], ks=P[4], vs=P[5], table=P[6], start=P[7], count=None, batch=1, tokens=2, heads=2, dim=64, page=16,
           pages=4, columns=4, ldt=4, st=ST, t=BF16):
    return status("ds_kv_cache_fp4_append", k, v, kc, vc, ks, vs, table, start, count, batch, tokens, heads, dim, page, pages, columns, ldt, st, st,
                  t, None)


def read(k=P[0], v=P[1], kc=P[2], vc=P[3], ks=P[4], vs=P[5], table=P[6], start=P[7], count=None, batch=1, tokens=2, heads=2, dim=64, page=16,
         pages=4, columns=4, ldt=4, st=ST, t=BF16):
    return status("ds_kv_cache_fp4_read", kc, vc, ks, vs, table, start, count, k, v, batch, tokens, heads, dim, page, pages, columns, ldt, st, st,
                  t, None)


def attention(q=P[0], kc=P[2], vc=P[3], ks=P[4], vs=P[5], table=P[6], length=P[7], count=None, o=P[8], batch=1, tokens=2, heads=2, group=2,
              dim=64, page=16, pages=4, columns=4, ldt=4, st=ST, scale=0.1, window=0, t=BF16):
    return status("ds_attention_fp4", q, kc, vc, ks, vs, table, length, count, o, batch, tokens, heads, group, dim, page, pages, columns, ldt, st, st,
                  scale, window, t, None, 0, None)


CACHE = [(SHAPE, dict(batch=-1)), (SHAPE, dict(tokens=-1)), (SHAPE, dict(heads=0)), (SHAPE, dict(dim=0)), (SHAPE, dict(pages=0)), (SHAPE, dict(columns=0)),
         (UNSUP, dict(dim=72)), (UNSUP, dict(dim=272)), (UNSUP, dict(page=8)), (UNSUP, dict(page=256)), (UNSUP, dict(page=48)), (ARG, dict(ldt=3)),
         (NULLP, dict(kc=None)), (NULLP, dict(vc=None)), (NULLP, dict(ks=None)), (NULLP, dict(vs=None)), (NULLP, dict(table=None)),
         (NULLP, dict(st=None)), (ARG, dict(t=E4M3)), (ARG, dict(kc=P[2] + 8)), (ARG, dict(vs=P[5] + 4)), (ARG, {}),
         (ARG, dict(st=strides(1024, -128, 64))), (UNSUP, dict(batch=2, ldt=2 ** 61)), (UNSUP, dict(batch=2, st=strides(2 ** 61, 128, 64))),
         (UNSUP, dict(columns=2 ** 27 - 1, ldt=2 ** 30)), (UNSUP, dict(columns=2 ** 60, ldt=2 ** 60))]
MOVES = CACHE + [(NULLP, dict(k=None)), (NULLP, dict(v=None)), (NULLP, dict(start=None)), (ARG, dict(k=P[2])), (ARG, dict(vc=P[0])),
                 (UNSUP, dict(tokens=2 ** 24, heads=65535)), (UNSUP, dict(batch=2 ** 20, tokens=2 ** 10))]


@pytest.mark.parametrize("want,kw", MOVES + [(ARG, dict(vc=P[2]))])
def test_append(want, kw):
    assert append(**kw) == want


@pytest.mark.parametrize("want,kw", MOVES + [(ARG, dict(v=P[0]))])
def test_read(want, kw):
    assert read(**kw) == want


@pytest.mark.parametrize("want,kw", CACHE + [(NULLP, dict(q=None)), (NULLP, dict(o=None)), (NULLP, dict(length=None)), (ARG, dict(o=P[0])),
                                             (ARG, dict(t=F32)), (SHAPE, dict(group=0)), (ARG, dict(window=-1)), (ARG, dict(scale=float("nan"))),
                                             (UNSUP, dict(batch=70000)), (NULLP, dict(columns=4096, ldt=4096, tokens=1)),
                                             (UNSUP, dict(tokens=2 ** 24, group=64))])
def test_attention(want, kw):
    assert attention(**kw) == want


def test_wrappers_refuse_host_tensors():
    x, i = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    cache = ops.kv_cache_fp4(4, 2, 16, 64, "cpu")
    f = ops.rotary_frequencies(32, device="cpu")
    for call in (lambda: ops.rotary_norm(x, x, i[None], f), lambda: ops.rotary_norm_backward(x, x, x, x, i[None], f),
                 lambda: ops.kv_cache_fp4_append(x, x, *cache, i[None], i), lambda: ops.kv_cache_fp4_read(*cache, i[None], i, 4),
                 lambda: ops.attention_fp4(x, *cache, i[None], i)):
        with pytest.raises(TypeError):
            call()
    for bad in ((4, 2, 24, 64), (4, 2, 32, 60), (0, 2, 32, 64), (4, 2, 32, 272)):
        with pytest.raises(ValueError):
            ops.kv_cache_fp4(*bad, "cpu")
    with pytest.raises(ValueError):
        ops.rotary_frequencies(0, device="cpu")
