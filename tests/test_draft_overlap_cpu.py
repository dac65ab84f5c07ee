"""Results that would overlap one another, or what is still read, are refused on the host.  Where a GPU is there, nothing is
called with these addresses: what fails no check would be launched."""
import pytest
import torch

from paper_2609_34060_amd import kvc
from tests.test_draft_abi_cpu import FAKE, Call, sets

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="addresses that are none")
S, X = kvc.KVC_ERR_SHAPE, kvc.KVC_ERR_ALIAS


def apart(c):
    for i, x in enumerate(("parents", "tokens", "target", "draft", "uniforms", "last", "path", "counts", "chosen")):
        setattr(c.draft, x, FAKE + 0x1000000 * (i + 1))


def strides(token, head):
    return lambda c: (sets("q.out_token_stride", token)(c), sets("q.out_head_stride", head)(c))


ROTATE = [(strides(128, 128), S), (strides(256, 128), S), (strides(128, 256), S), (strides(1016, 128), S),
          (strides(128, 632), S), (sets("k.out", FAKE + 0x10000), X), (sets("k.out", FAKE), X),
          (sets("q.out", FAKE + 0x20000), X)]
VERIFY = [(lambda c, a=a, b=b: setattr(c.draft, a, getattr(c.draft, b)), X)
          for a, b in (("path", "parents"), ("path", "tokens"), ("path", "uniforms"), ("path", "target"), ("path", "draft"),
                       ("counts", "chosen"), ("counts", "path"), ("chosen", "path"), ("counts", "last"),
                       ("chosen", "last"), ("counts", "parents"), ("chosen", "tokens"))]


@pytest.mark.parametrize("at", range(len(ROTATE)))
def test_rotated_rows(at):
    c = Call()
    ROTATE[at][0](c)
    assert c.rotate() == ROTATE[at][1]


@pytest.mark.parametrize("at", range(len(VERIFY)))
def test_verified(at):
    c = Call()
    apart(c)
    VERIFY[at][0](c)
    assert c.verify() == VERIFY[at][1]


@pytest.mark.parametrize("token, head", [(1024, 128), (128, 640), (2048, 256), (136, 680)])
def test_layouts_that_are_apart(token, head):
    """5 rows of 8 heads, tokens or heads outermost: no check of the host's refuses them (a launch fails where no GPU is)."""
    c = Call()
    strides(token, head)(c)
    assert c.rotate() not in (S, X)
    apart(c)
    assert c.verify() not in (S, X)
