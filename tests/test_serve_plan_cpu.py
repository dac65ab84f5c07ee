"""The workspace that kvc_attend asks for, worked out on the host: bounded for every step, and enough for every window."""
import ctypes

import pytest

from paper_2609_34060_amd import kvc

FAKE = 0x10000


def need(dtype, d, H, heads, n, N, max_new, ctx):
    pools = (ctypes.c_void_p * 1)(FAKE)
    at = ctypes.cast(pools, ctypes.POINTER(ctypes.c_void_p))
    cache = kvc.kvc_cache(dtype, 1, H, d, 16, 1 << 20, 16 * H * d, H * d, d, at, at, 0, 0, None)
    step = kvc.kvc_step(n, N, max_new, ctx, -(-ctx // 16), 0, FAKE, FAKE, None, FAKE)
    return kvc.load().kvc_attend_workspace_bytes(ctypes.addressof(cache), ctypes.addressof(step), heads)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,heads", [(1, 1), (2, 16), (4, 28), (8, 32), (8, 64)])
@pytest.mark.parametrize("new", [65, 257, 300, 512, 1500, 4096, 32768])
@pytest.mark.parametrize("ctx", [257, 4096, 32768, 1 << 20])
@pytest.mark.parametrize("seqs", [1, 3, 64])
def test_chunks_of_float32(d, H, heads, new, ctx, seqs):
    """Chunks of more than 256 rows a sequence are cut only to fill the chip with 256 workgroups of 16 rows: 8192 rows of
    parts at most, however long the context is.  Shorter ones into ranges of 1280 keys: a tenth of the keys and values that
    their sequences may hold."""
    got = need(kvc.KVC_F32, d, H, heads, seqs, seqs * new, new, ctx)
    fill = 8192 * (4 * d + 8)
    if new * heads // H > 256:
        assert got <= fill
    else:
        assert got <= max(fill, seqs * (ctx + 1280) * H * 2 * 4 * d * 0.11)


@pytest.mark.parametrize("dtype", [kvc.KVC_BF16, kvc.KVC_I8])
@pytest.mark.parametrize("new", [1, 5, 65, 300, 4096])
@pytest.mark.parametrize("ctx", [257, 4096, 32768, 1 << 20])
@pytest.mark.parametrize("seqs", [1, 64])
def test_others(dtype, new, ctx, seqs):
    """16-bit and 8-bit caches: 512 workgroups of 128 rows, or one tile's 16 rows a range of 1280 keys."""
    got = need(dtype, 128, 8, 32, seqs, seqs * new, new, ctx)
    assert got <= max(520 * 512 * 256 * 2, 520 * seqs * 32 * new * (ctx // 1280 + 1) if 4 * new <= 16 else 0)


@pytest.mark.parametrize("scale,refused", [(2.0 ** 127, False), (-2.0 ** 127, False), (2.5e38, True), (-3.4e38, True),
                                           (0.0, False), (1e-45, False)])
def test_scales_in_units_of_log2(scale, refused):
    """A scale is refused where its scores, which are kept in units of log2, would be infinite or NaN throughout."""
    pools = (ctypes.c_void_p * 1)(FAKE)
    at = ctypes.cast(pools, ctypes.POINTER(ctypes.c_void_p))
    cache = kvc.kvc_cache(kvc.KVC_BF16, 1, 2, 128, 16, 64, 16 * 256, 256, 128, at, at, 0, 0, None)
    step = kvc.kvc_step(1, 0, 0, 10, 1, 0, FAKE, FAKE, None, FAKE)
    query = kvc.kvc_query(kvc.KVC_BF16, 8, 1, 0, scale, 0, FAKE, 1024, 128, FAKE, 1024, 128, None)
    got = kvc.load().kvc_attend(ctypes.addressof(cache), None, ctypes.addressof(step), bytes(query), 0, None, 0, None)
    assert got == (kvc.KVC_ERR_SHAPE if refused else kvc.KVC_OK)
