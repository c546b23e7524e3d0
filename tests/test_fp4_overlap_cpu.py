"""Outputs that lie between another output's vectors are refused, whole ones behind each other are not (no device access)."""
import pytest

from paper_1905_13298_amd import _native

from .test_fp4_abi_cpu import P, rotary, rotary_grad, strides

TOKEN = strides(2 * 4 * 64, 4 * 64, 64)           # 2 heads of q and 2 of k, 64 elements each, in a token's row of 16-bit floats
PART = 2 * 64 * 2


@pytest.mark.parametrize("base,call", [(P[6], lambda k: rotary(qo=P[6], ko=k, so=TOKEN, sko=TOKEN)),
                                       (P[8], lambda k: rotary_grad(dq=P[8], dk=k, sdq=TOKEN, sdk=TOKEN))])
def test_parts_of_one_buffer(base, call):
    # Two tokens of q end 6 vectors on.
    for at, overlaps in ((PART, True), (6 * 64 * 2 - 2, True), (6 * 64 * 2, False), (4096, False)):
        assert call(base + at) == 3                  # (DS_ERR_INVALID_ARG in the end: not device memory)
        assert (b"overlaps" in _native.lib().ds_last_error_message()) is overlaps, at
