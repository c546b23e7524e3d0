"""The 8-bit operators' checks at the ends of their ranges, without a GPU: what a launch, an
offset or a count of bytes cannot hold is refused as such before the device is looked at."""
import ctypes

import pytest

from .test_fp8_abi_cpu import ARG, E4M3, P, SHAPE, SMALL, UNSUP, append, attention, grad, linear, norm, status  # noqa: F401


def quantize(rows, cols, ld):
    return status("ds_quantize_fp8", P[0], None, P[1], P[2], rows, cols, cols, 0, ld, (cols + 127) // 128, 2, None)


@pytest.mark.parametrize("rows,cols,want", [
    (2 ** 26 - 4, 256, ARG), (2 ** 26, 256, UNSUP), (2 ** 24 - 1, 2048, ARG), (2 ** 24, 2048, UNSUP), (2 ** 23 - 1, 4096, ARG),
    (2 ** 23, 4096, UNSUP), (2 ** 22 - 1, 32768, ARG), (2 ** 22, 32768, UNSUP)])
def test_norm_rows_of_a_launch(rows, cols, want):
    """(ARG: accepted up to the look at the pointers, which are none.)"""
    assert norm(rows=rows, cols=cols, ldx=cols, ldr=cols, ldh=cols, ldy=cols, lds=cols // 128) == want


def test_quantiser_scales_of_a_launch():
    assert quantize(2 ** 28 - 16, 16, 16) == ARG and quantize(2 ** 28, 16, 16) == UNSUP
    call = lambda cols: status("ds_quantize_weights_fp8", P[0], P[1], P[2], 1, cols, cols, (cols + 15) // 16 * 16, 2 ** 24, 2, None)  # noqa: E731
    assert call(2 ** 31 - 256) == ARG and call(2 ** 31 - 100) == UNSUP


def test_product_rows_out_of_the_tiles_reach():
    far = 2 ** 22 + 16
    assert linear(m=64 * 65535, ldw=far) == ARG and linear(m=64 * 65535 + 1, ldw=far) == UNSUP
    assert linear(m=64 * 65535 + 1) == ARG
    n = 2 ** 22 + 1
    size = dict(n=n, k=16, lddy=n + 15, ldds=n // 128 + 1, ldw=16, ldws=1, lddx=16, size=1 << 40)
    assert grad(m=64 * 65535, **size) == ARG and grad(m=64 * 65535 + 1, **size) == UNSUP


def test_append_pages_of_a_launch():
    assert append(batch=2 ** 20, tokens=16 * 14) == ARG and append(batch=2 ** 20, tokens=16 * 15 + 2) == UNSUP


def test_columns_times_page_of_a_table():
    """Key positions are 32-bit numbers, some steps past the last one."""
    for call in (append, attention):
        assert call(columns=(2 ** 31 - 4096) // 16, ldt=2 ** 30) != UNSUP
        assert call(columns=2 ** 27 - 1, ldt=2 ** 30) == UNSUP         # 2^31 - 16 keys
        assert call(columns=2 ** 60, ldt=2 ** 60) == UNSUP             # 2^64 keys
        assert call(columns=2 ** 62, ldt=2 ** 62, page=128) == UNSUP


FAR = 2 ** 61      # elements between rows: two rows of 16-bit elements are 2^62 bytes apart


@pytest.mark.parametrize("by", ["ldx", "ldr", "ldh", "ldy", "lds"])
def test_norm_strides_past_what_bytes_count(by):
    assert norm(**{by: FAR * 2 if by in ("ldy", "lds") else FAR}) == UNSUP
    assert norm(rows=1, **{by: FAR}) == ARG        # a single row goes nowhere


def test_other_strides_past_what_bytes_count():
    assert status("ds_rms_norm_backward", *P[:7], 4, 256, 256, FAR, 256, 256, 2, 2, P[8], 1 << 20, None) == UNSUP
    assert status("ds_quantize_fp8", P[0], None, P[1], P[2], 4, 256, FAR, 0, 256, 2, 2, None) == UNSUP
    assert status("ds_quantize_weights_fp8", P[0], P[1], P[2], 4, 256, 256, FAR * 2, 2, 2, None) == UNSUP
    assert status("ds_shift_weights_to_fp8", P[0], P[1], 4, 256, FAR * 2, 0, None) == UNSUP
    assert linear(ldy=FAR) == UNSUP and linear(ldw=FAR) == UNSUP and linear(ldxs=FAR * 3) == UNSUP
    assert grad(lddx=FAR) == UNSUP and grad(ldws=FAR * 2) == ARG       # (one row of scales)
    for where in range(3):
        size = [1024, 128, 64]
        size[where] = FAR
        kept = (ctypes.c_int64 * 3)(*size)
        st = ctypes.cast(kept, ctypes.c_void_p)
        assert append(st=st, batch=2) == UNSUP and attention(st=st, batch=2) == UNSUP
    assert append(batch=2, ldt=FAR) == UNSUP and attention(batch=2, ldt=FAR) == UNSUP
