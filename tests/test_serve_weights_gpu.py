"""Weights of single tokens and short lists of rows reach the values with 16 bits: what is left is the result's rounding.

Bounds, with u = 2^-24, A the weighted mean of |v|, and a score's error e = (d + 4) u mass + 4 u |s|: weights are off by a
factor of at most 1 + 2 e + 8 u, and by 2^-15 and 2^-20 for their two bfloat16 terms; sums over n tokens by n u A; the result's
rounding is 2^-8 |out|."""
import numpy as np
import pytest

from oracle import serve_oracle as SO
from paper_2609_34060_amd import kvc
from tests.test_serve_gpu import Setup

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("i8", 128), ("bf16", 64), ("i8", 64)])
@pytest.mark.parametrize("new,ctx,Hq", [([1, 1, 1], [40, 300, 1000], 8), ([1], [4000], 2), ([1], [100], 32), ([3, 1], [700, 60], 8)])
def test_results_are_rounded_once(kind, d, new, ctx, Hq):
    su = Setup(new, ctx, d=d, cache=kind)
    assert max(new) * Hq // su.H <= 16
    q = su.queries(Hq)
    got = kvc.kvc_attend(su.cache(), su.step(), q).double().cpu().numpy()
    k, v = su.values()
    ref, _, mean, mass, peak, n = SO.attend(q.double().cpu().numpy(), k, v, su.new, su.ctx, su.offs, su.tables, d ** -0.5,
                                            True, 0)
    e = (d + 4) * U * mass + 4 * U * peak
    bound = (2 * e + (8 + n) * U + 2.0 ** -15 + 2.0 ** -20)[..., None] * mean * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(ref) + 1e-30
    assert np.all(np.abs(got - ref) <= bound), np.max(np.abs(got - ref) / bound)
