"""kvc_rotate takes up to 2^30 tokens: its launches count them in 32 bits, a step of 2^23 at a time."""
import ctypes

import pytest

from paper_2609_34060_amd import kvc

FAKE = 0x7F0000001000


def rotate(rows, heads):
    freq = (ctypes.c_double * 32)(*[0.5] * 32)
    r = kvc.kvc_rotary(kvc.KVC_BF16, rows, 64, kvc.KVC_ROPE_HALF, 64, 0, 1.0, ctypes.addressof(freq), None)
    h = kvc.kvc_heads(heads, 0, FAKE, 0, 0, FAKE + (1 << 40), 64, 64)
    return kvc.load().kvc_rotate(bytes(r), bytes(h), None, None)


@pytest.mark.parametrize("rows", [2 ** 31 - 1, 2 ** 31 - 2 ** 23, 2 ** 30 + 1])
def test_more_rows_are_refused(rows):
    assert rotate(rows, 1) == rotate(rows, 0) == kvc.KVC_ERR_SHAPE


def test_as_many_are_taken():
    assert rotate(2 ** 30, 0) == kvc.KVC_OK                  # (nothing to do)
    assert rotate(2 ** 30, 1) == kvc.KVC_ERR_NULL_ARG        # (the positions: the call came so far)
