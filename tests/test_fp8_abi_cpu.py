"""Argument checks of the 8-bit decoder operators that need no GPU: they run before any
device access, so bad sizes, types, strides and pointers are refused with the documented
status."""
import ctypes

import pytest
import torch

from paper_1905_13298_amd import _native, ops

OK, NULLP, SHAPE, ARG, SMALL, CODE, HIP, UNSUP = range(8)
P = [0x100000 * (i + 1) for i in range(12)]       # never dereferenced
F32, F16, BF16, E4M3, E5M2 = range(5)
STRIDES = ctypes.cast((ctypes.c_int64 * 3)(1024, 128, 64), ctypes.c_void_p)


def status(name, *args):
    return getattr(_native.lib(), name)(*args)


def norm(x=P[0], r=P[1], w=P[2], y=P[3], s=P[4], h=P[5], rstd=P[6], rows=4, cols=256, ldx=256, ldr=256, ldh=256, ldy=256, lds=2,
         eps=1e-6, t=BF16, wt=BF16, yt=E4M3):
    return status("ds_rms_norm", x, r, w, y, s, h, rstd, rows, cols, ldx, ldr, ldh, ldy, lds, eps, t, wt, yt, None)


@pytest.mark.parametrize("want,kw", [
    (NULLP, dict(x=None)), (NULLP, dict(w=None)), (NULLP, dict(y=None)), (NULLP, dict(h=None)), (NULLP, dict(s=None)),
    (ARG, dict(r=None)), (SHAPE, dict(rows=-1)), (SHAPE, dict(cols=0)), (UNSUP, dict(cols=65537)), (ARG, dict(t=E4M3)), (ARG, dict(t=9)),
    (ARG, dict(wt=F16)), (ARG, dict(yt=F16)), (ARG, dict(yt=E5M2)), (ARG, dict(eps=-1.0)), (ARG, dict(eps=float("nan"))),
    (ARG, dict(ldx=255)), (ARG, dict(ldr=255)), (ARG, dict(ldh=255)), (ARG, dict(ldy=255)), (ARG, dict(ldy=264)), (ARG, dict(y=P[3] + 8)),
    (ARG, dict(lds=1)), (ARG, dict(yt=BF16, ldy=255)), (ARG, dict(h=P[0])), (ARG, dict(y=P[1])), (UNSUP, dict(rows=2 ** 31)),
    (ARG, {}),                                     # not device memory
])
def test_norm(want, kw):
    assert norm(**kw) == want


def test_calls_without_rows_do_nothing():
    assert norm(rows=0) == OK
    assert norm(rows=0, x=None, y=None, s=None, h=None, r=None) == OK
    assert status("ds_quantize_fp8", None, None, None, None, 0, 8, 8, 0, 16, 1, BF16, None) == OK
    assert linear(m=0, x=None, y=None) == OK
    assert grad(m=0, dy=None, dx=None, scratch=None, size=0) == OK
    assert append(batch=0, k=None, v=None) == OK and append(tokens=0) == OK
    assert attention(batch=0, q=None, o=None) == OK and attention(tokens=0) == OK


def norm_grad(dy=P[0], h=P[1], w=P[2], rstd=P[3], dh=P[4], dx=P[5], dw=P[6], rows=4, cols=256, ld=(256,) * 4, t=BF16, wt=F32,
              scratch=P[7], size=1 << 20):
    return status("ds_rms_norm_backward", dy, h, w, rstd, dh, dx, dw, rows, cols, *ld, t, wt, scratch, size, None)


@pytest.mark.parametrize("want,kw", [
    (NULLP, dict(dy=None)), (NULLP, dict(h=None)), (NULLP, dict(w=None)), (NULLP, dict(rstd=None)), (NULLP, dict(dx=None)),
    (NULLP, dict(scratch=None)), (SMALL, dict(size=4095)), (SHAPE, dict(rows=-1)), (SHAPE, dict(cols=-1)), (UNSUP, dict(cols=65537)), (ARG, dict(t=E5M2)),
    (ARG, dict(wt=F16)), (ARG, dict(ld=(255, 256, 256, 256))), (ARG, dict(ld=(256, 255, 256, 256))),
    (ARG, dict(ld=(256, 256, 255, 256))), (ARG, dict(ld=(256, 256, 256, 255))), (ARG, dict(dx=P[0])), (ARG, dict(scratch=P[1])),
])
def test_norm_gradient(want, kw):
    assert norm_grad(**kw) == want


def test_scratch_sizes():
    lib = _native.lib()
    assert lib.ds_rms_norm_backward_scratch_bytes(0, 8) == 0 and lib.ds_rms_norm_backward_scratch_bytes(4, -1) == 0
    assert lib.ds_rms_norm_backward_scratch_bytes(4, 256) == 4 * 256 * 4
    assert lib.ds_linear_fp8_backward_data_scratch_bytes(0, 8, 8) == 0
    assert lib.ds_attention_fp8_scratch_bytes(0, 1, 1, 1, 64, 16, 4) == 0
    assert lib.ds_attention_fp8_scratch_bytes(1, 1, 8, 4, 128, 64, 4096) > 0


@pytest.mark.parametrize("want,args", [
    (NULLP, (None, None, P[1], P[2], 4, 256, 256, 0, 256, 2, BF16)), (NULLP, (P[0], None, None, P[2], 4, 256, 256, 0, 256, 2, BF16)),
    (NULLP, (P[0], None, P[1], None, 4, 256, 256, 0, 256, 2, BF16)), (SHAPE, (P[0], None, P[1], P[2], -4, 256, 256, 0, 256, 2, BF16)),
    (ARG, (P[0], None, P[1], P[2], 4, 256, 255, 0, 256, 2, BF16)), (ARG, (P[0], P[3], P[1], P[2], 4, 256, 256, 255, 256, 2, BF16)),
    (ARG, (P[0], None, P[1], P[2], 4, 256, 256, 0, 250, 2, BF16)), (ARG, (P[0], None, P[1], P[2], 4, 256, 256, 0, 256, 1, BF16)),
    (ARG, (P[0], None, P[1], P[2], 4, 256, 256, 0, 256, 2, E4M3)), (ARG, (P[0], None, P[0], P[2], 4, 256, 256, 0, 256, 2, BF16)),
])
def test_quantize(want, args):
    assert status("ds_quantize_fp8", *args, None) == want


def test_quantize_weights_and_shift_weights():
    call = lambda *a: status("ds_quantize_weights_fp8", *a, None)  # noqa: E731
    assert call(None, P[1], P[2], 4, 256, 256, 256, 2, BF16) == NULLP
    assert call(P[0], P[1], P[2], 0, 256, 256, 256, 2, BF16) == SHAPE
    assert call(P[0], P[1], P[2], 4, 256, 200, 256, 2, BF16) == ARG
    assert call(P[0], P[1], P[2], 4, 256, 256, 256, 1, BF16) == ARG
    assert call(P[0], P[1], P[2], 128 * 65536, 16, 16, 16, 1, BF16) == UNSUP
    call = lambda *a: status("ds_shift_weights_to_fp8", *a, None)  # noqa: E731
    assert call(None, P[1], 4, 256, 256, 0) == NULLP
    assert call(P[0], P[1], 0, 256, 256, 0) == SHAPE
    assert call(P[0], P[1], 4, 256, 256, 1) == ARG
    assert call(P[0], P[1], 4, 256, 256, 6 << 8) == ARG
    assert call(P[0], P[1], 4, 256, 240, 0) == ARG
    assert call(P[0], P[1], 65536, 256, 256, 0) == UNSUP


def linear(x=P[0], xs=P[1], w=P[2], ws=P[3], bias=None, y=P[4], m=4, n=32, k=256, ldx=256, ldxs=2, ldw=256, ldws=2, ldy=32, wt=E4M3, yt=BF16):
    return status("ds_linear_fp8", x, xs, w, ws, bias, y, m, n, k, ldx, ldxs, ldw, ldws, ldy, wt, yt, None)


def grad(dy=P[0], ds=P[1], w=P[2], ws=P[3], dx=P[4], m=4, n=32, k=256, lddy=32, ldds=1, ldw=256, ldws=2, lddx=256, wt=E4M3, t=BF16,
         scratch=P[5], size=1 << 24):
    return status("ds_linear_fp8_backward_data", dy, ds, w, ws, dx, m, n, k, lddy, ldds, ldw, ldws, lddx, wt, t, scratch, size, None)


@pytest.mark.parametrize("want,kw", [
    (NULLP, dict(x=None)), (NULLP, dict(xs=None)), (NULLP, dict(w=None)), (NULLP, dict(ws=None)), (NULLP, dict(y=None)),
    (SHAPE, dict(m=-1)), (SHAPE, dict(n=0)), (SHAPE, dict(k=0)), (UNSUP, dict(m=2 ** 26)), (ARG, dict(wt=BF16)), (ARG, dict(yt=E4M3)),
    (ARG, dict(ldx=255)), (ARG, dict(ldx=264)), (ARG, dict(ldw=128)), (ARG, dict(x=P[0] + 1)), (ARG, dict(w=P[2] + 8)), (ARG, dict(ldxs=1)),
    (ARG, dict(ldws=1)), (ARG, dict(ldy=31)), (ARG, dict(y=P[0])), (ARG, {}),
])
def test_linear(want, kw):
    assert linear(**kw) == want


@pytest.mark.parametrize("want,kw", [
    (NULLP, dict(dy=None)), (NULLP, dict(dx=None)), (NULLP, dict(w=None)), (SHAPE, dict(k=-1)), (ARG, dict(lddy=16)), (ARG, dict(lddx=255)),
    (ARG, dict(ldw=250)), (ARG, dict(ldds=0)), (ARG, dict(wt=0)), (ARG, dict(t=4)), (ARG, dict(dx=P[2])), (ARG, {}),
])
def test_linear_gradient(want, kw):
    assert grad(**kw) == want


def append(k=P[0], v=P[1], kc=P[2], vc=P[3], ks=P[4], vs=P[5], table=P[6], start=P[7], count=None, batch=1, tokens=2, heads=2, dim=64, page=16,
           pages=4, columns=4, ldt=4, st=STRIDES, t=BF16):
    return status("ds_kv_cache_append", k, v, kc, vc, ks, vs, table, start, count, batch, tokens, heads, dim, page, pages, columns, ldt, st, st, t, None)


def attention(q=P[0], kc=P[2], vc=P[3], ks=P[4], vs=P[5], table=P[6], length=P[7], count=None, o=P[8], batch=1, tokens=2, heads=2, group=2,
              dim=64, page=16, pages=4, columns=4, ldt=4, st=STRIDES, scale=0.1, window=0, t=BF16):
    return status("ds_attention_fp8", q, kc, vc, ks, vs, table, length, count, o, batch, tokens, heads, group, dim, page, pages, columns, ldt, st, st,
                  scale, window, t, None, 0, None)


CACHE = [(SHAPE, dict(batch=-1)), (SHAPE, dict(tokens=-1)), (SHAPE, dict(heads=0)), (SHAPE, dict(dim=0)), (SHAPE, dict(pages=0)), (SHAPE, dict(columns=0)),
         (UNSUP, dict(dim=72)), (UNSUP, dict(dim=272)), (UNSUP, dict(page=8)), (UNSUP, dict(page=256)), (UNSUP, dict(page=48)), (ARG, dict(ldt=3)),
         (NULLP, dict(kc=None)), (NULLP, dict(vc=None)), (NULLP, dict(ks=None)), (NULLP, dict(vs=None)), (NULLP, dict(table=None)),
         (NULLP, dict(st=None)), (ARG, dict(t=E4M3)), (ARG, {}),
         (ARG, dict(st=ctypes.cast((ctypes.c_int64 * 3)(1024, -128, 64), ctypes.c_void_p)))]


@pytest.mark.parametrize("want,kw", CACHE + [(NULLP, dict(k=None)), (NULLP, dict(v=None)), (NULLP, dict(start=None)), (ARG, dict(k=P[2])),
                                             (ARG, dict(vc=P[2]))])
def test_append(want, kw):
    assert append(**kw) == want


@pytest.mark.parametrize("want,kw", CACHE + [(NULLP, dict(q=None)), (NULLP, dict(o=None)), (NULLP, dict(length=None)), (ARG, dict(o=P[0])),
                                             (ARG, dict(t=F32)), (SHAPE, dict(group=0)), (ARG, dict(window=-1)), (ARG, dict(scale=float("nan"))),
                                             (UNSUP, dict(batch=70000)), (NULLP, dict(columns=4096, ldt=4096, tokens=1))])
def test_attention(want, kw):
    assert attention(**kw) == want


def test_wrappers_refuse_host_tensors():
    x, i = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    x8 = x.to(torch.float8_e4m3fn)
    sc = torch.full((4, 1), 127, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for f in (lambda: ops.rms_norm(x, x[0]), lambda: ops.quantize_fp8(x), lambda: ops.quantize_weights_fp8(x), lambda: ops.linear_fp8(x8, sc, x8, sc[:1]),
              lambda: ops.linear_fp8_backward_data(x8, sc, x8, sc[:1]), lambda: ops.rms_norm_backward(x, x, x[0], x[:, 0].float()),
              lambda: ops.attention_fp8(x[None, None], x8, x8, sc, sc, i[None], i)):
        with pytest.raises(TypeError):
            f()
    with pytest.raises(ValueError):
        ops.kv_cache(4, 2, 24, 64, "cpu")
    with pytest.raises(ValueError):
        ops.kv_cache(4, 2, 32, 60, "cpu")
