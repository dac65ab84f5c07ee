"""What each of the two attentions asks for by itself: kvc_attend does not pay for the ranges that only trees are cut into."""
import ctypes

import pytest

from paper_2609_34060_amd import kvc
from tests.tall_trees import plan

FAKE = 0x10000
KINDS = {"f32": kvc.KVC_F32, "bf16": kvc.KVC_BF16, "i8": kvc.KVC_I8}


def descriptors(kind, d, H, n, N, max_new, ctx):
    pools = (ctypes.c_void_p * 1)(FAKE)
    at = ctypes.cast(pools, ctypes.POINTER(ctypes.c_void_p))
    cache = kvc.kvc_cache(KINDS[kind], 1, H, d, 16, 1 << 20, 16 * H * d, H * d, d, at, at, 0, 0, None)
    return cache, kvc.kvc_step(n, N, max_new, ctx, -(-ctx // 16), 0, FAKE, FAKE, None, FAKE)


def needs(cache, step, heads):
    c, s, lib = ctypes.addressof(cache), ctypes.addressof(step), kvc.load()
    return (lib.kvc_attend_call_workspace_bytes(c, s, heads, 0), lib.kvc_attend_call_workspace_bytes(c, s, heads, 1),
            lib.kvc_attend_workspace_bytes(c, s, heads))


@pytest.mark.parametrize("kind", ["f32", "bf16", "i8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seqs,new,ctx", [(1, 1, 100), (1, 1, 32768), (64, 1, 16384), (64, 8, 16384), (64, 64, 16384),
                                          (8, 512, 4096), (16, 300, 32768), (300, 8, 2000), (1, 4096, 4096)])
def test_each_and_both(kind, d, seqs, new, ctx):
    cache, step = descriptors(kind, d, 8, seqs, seqs * new, new, ctx)
    own, tree, both = needs(cache, step, 32)
    assert own == plan(kind, seqs, seqs * new, new, ctx, ctx, 8, 4, d, False).most_bytes
    assert tree == plan(kind, seqs, seqs * new, new, ctx, ctx, 8, 4, d, True).most_bytes
    assert both == max(own, tree)


@pytest.mark.parametrize("kind", ["bf16", "i8"])
@pytest.mark.parametrize("seqs,new,ctx", [(8, 512, 4096), (64, 64, 16384), (64, 8, 16384), (8, 256, 8192)])
def test_chunks_that_are_not_cut_need_nothing(kind, seqs, new, ctx):
    cache, step = descriptors(kind, 128, 8, seqs, seqs * new, new, ctx)
    own, tree, _ = needs(cache, step, 32)
    assert own == 0 and tree > 0


def test_where_nothing_can_be_told():
    cache, step = descriptors("bf16", 128, 8, 1, 1, 1, 32768)
    c, s, call = ctypes.addressof(cache), ctypes.addressof(step), kvc.load().kvc_attend_call_workspace_bytes
    assert call(c, s, 32, 0) > 0 and call(c, s, 32, 1) > 0
    for args in ((None, s, 32, 0), (c, None, 32, 0), (c, s, 0, 0), (c, s, 7, 1), (c, s, 32, 2), (c, s, 32, -1)):
        assert call(*args) == 0
    step.max_context = -1
    assert call(c, s, 32, 0) == call(c, s, 32, 1) == 0
