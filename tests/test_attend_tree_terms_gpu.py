"""kvc_attend_tree's weights over lists of up to 32 rows: two bfloat16 terms, and so 2^-16 of themselves, where one would be
2^-8 off.

Keys of two kinds, half of each: scores 0 (weight 1) and s, of weight w = e^s, which lies nearly half a step between two
bfloat16 numbers; values of the former -w' and of the latter 1, with w' the bfloat16 next to w, so that the result nearly
cancels.  With one term it is off by |w - w'| / (1 + w); the bounds, with u = 2^-24, n keys and A the weighted mean of |v|: one
product of a score counts (mass = |s|), so e = (d + 4) u |s| + 4 u |s|, and the quotient is off by (4 e + 16 u + 2 n u) A, for
the two terms by 2^-8 2^-8 A, for the result's rounding by 2^-8 of it."""
import numpy as np
import pytest
import torch

from paper_2609_34060_amd import kvc
from tests.draft_helpers import DEV, i64
from tests.tall_trees import plan
from tests.test_serve_gpu import U, Setup

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.tensor(x, dtype=torch.float64).to(torch.bfloat16).double().item()


def score():
    """Of the bfloat16 numbers in (-1, -1/2), the one whose exponential is the farthest from its own bfloat16."""
    return max((-1.0 + i / 256 for i in range(1, 128)), key=lambda s: abs(np.exp(s) - bf16(np.exp(s))))


# (sequences, new tokens, keys, heads, group): one 16-row tile and two; one range of keys, several, and shares
STEPS = [(1, 4, 96, 2, 4), (1, 8, 96, 2, 4), (1, 8, 4096, 1, 4), (3, 2, 96, 2, 8), (3, 5, 1024, 2, 5), (24, 8, 1024, 2, 4),
         (24, 4, 1024, 2, 7), (1, 32, 384, 1, 1), (1, 16, 384, 1, 1)]


@pytest.mark.parametrize("kind", ["bf16", "i8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seqs,new,keys,H,g", STEPS)
def test_two_terms(kind, d, seqs, new, keys, H, g):
    su = Setup([new] * seqs, [keys + new] * seqs, H=H, d=d, cache=kind, bs=16)
    p = plan(kind, seqs, seqs * new, new, keys + new, keys + new, H, g, d)
    assert p.tile_rows == (16 if new * g <= 16 else 32)
    s, count = score(), keys
    w = np.exp(s)
    near = bf16(w)
    # an 8-bit value is a code times its scale: the one term is of weight times scale, a power of two
    kv = su.pools
    kv.zero_()
    if kind == "i8":
        su.scales.fill_(2.0 ** -5)
    blocks = torch.from_numpy(su.tables).to(DEV)
    for i in range(seqs):
        place = torch.arange(keys + new, device=DEV)
        b, at = blocks[i][place // 16], place % 16
        odd, new_row = place % 2 == 1, place >= keys
        k0 = torch.where(odd, 32.0 if kind == "i8" else 1.0, 0.0)
        kv[0, 0, b, at, :, 0] = k0[:, None].to(kv.dtype)
        if kind == "i8":  # codes that stand in the ratio of w' and 1 as nearly as whole numbers do
            v = torch.where(odd, 127.0, -float(round(127 * near)))
        else:
            v = torch.where(odd, 1.0, -near)
        kv[1, 0, b, at] = torch.where(new_row, torch.zeros_like(v), v)[:, None, None].to(kv.dtype)
    one = 2.0 ** -5 if kind == "i8" else 1.0  # a code's worth
    hi, lo = (127.0 * one, -float(round(127 * near)) * one) if kind == "i8" else (1.0, -near)
    q = torch.zeros(su.N, H * g, d, dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = s
    masks = np.zeros((su.N, 1), np.uint64)  # the new tokens see the context alone
    got = kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks), q, scale=1.0).double()
    share = lambda x: (x * hi + lo) / (w + 1.0)  # for a weight x of the odd keys in the products
    want, mean = share(w), (w * hi + abs(lo)) / (w + 1.0)
    e = (d + 8) * U * abs(s)
    bound = (4 * e + (16 + 2 * count) * U + 2.0 ** -16) * mean + 2.0 ** -8 * abs(want)
    assert abs(share(near) - want) > 1.5 * bound  # (one term would show)
    assert bool(((got - want).abs() <= bound).all()), float((got - want).abs().max() / bound)
