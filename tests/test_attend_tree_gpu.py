"""kvc_attend_tree against the oracle in float64.

Bounds, with u = 2^-24, n keys and A the weighted mean of |v|: a score is off by e = (d + 4) u mass + 4 u |s| (d products
and sums of magnitudes `mass`, the scaling, the exponent's argument), a weight by a factor of 1 + 2 e + 8 u at most; sums
over n weights by n u; so the quotient by (4 e + 16 u + 2 n u) A.  A weight that goes into its product as a bfloat16 adds
2^-8 A, as the sum of two 2^-15 A; the result's rounding adds half a step, 2^-8 or u, of its magnitude.  lse is off by
2 e + n u + 8 u |lse| + 8 u."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from paper_2609_34060_amd import kvc
from tests.draft_helpers import DEV, TREES, i64, tree
from tests.test_serve_gpu import Setup

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def masks_of(su, kinds=TREES, seed=0, words=None):
    rng = np.random.default_rng(seed)
    words = max(1, -(-max(su.new) // 64)) if words is None else words
    return np.concatenate([DO.tree(tree(kinds[i % len(kinds)], q, rng), 0, words)[0] for i, q in enumerate(su.new)])


def check(su, Hq, masks, window=0, scale=None, layer=0, q=None, workspace=None):
    cache, step = su.cache(), su.step()
    q = su.queries(Hq) if q is None else q
    lse = torch.full((su.N, Hq), 77.0, device=DEV)
    out = torch.full((su.N, Hq, su.d), 77.0, dtype=su.rows, device=DEV)
    kvc.kvc_attend_tree(cache, step, i64(masks), q, out, lse=lse, layer=layer, scale=scale, window=window,
                        workspace=workspace)
    compare(su, Hq, masks, q, out, lse, window, scale, layer)
    return out, lse


def compare(su, Hq, masks, q, out, lse, window=0, scale=None, layer=0):
    k, v = su.values(layer)
    sc = su.d ** -0.5 if scale is None else scale
    ref, rlse, mean, mass, peak, n = DO.attend(q.double().cpu().numpy(), k, v, su.new, su.ctx, su.offs, su.tables, masks, sc,
                                               window)
    got, glse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    assert np.array_equal(np.isinf(ref), np.isinf(got) & (got == ref))
    half = U if su.kind == "f32" else 2.0 ** -8
    e = (su.d + 4) * U * mass + 4 * U * peak
    weight = (4 * e + (16 + 2 * n) * U + (0.0 if su.kind == "f32" else 2.0 ** -8))[..., None] * mean
    fin = np.isfinite(ref)
    err = np.where(fin, np.abs(np.where(fin, got, 0) - np.where(fin, ref, 0)), 0.0)
    bound = weight + half * np.abs(np.where(fin, ref, 0)) + 1e-30
    assert np.all(np.where(fin, err <= bound, True)), np.nanmax(err / bound)
    none = rlse == -np.inf
    assert np.array_equal(none, glse == -np.inf)
    assert not np.any(got[none])
    ok = np.isfinite(rlse)
    assert np.array_equal(np.isnan(rlse), np.isnan(glse))
    lerr = np.abs(np.where(ok, glse, 0) - np.where(ok, rlse, 0))
    assert np.all(np.where(ok, lerr <= 2 * e + n * U + 8 * U * np.abs(np.where(ok, rlse, 0)) + 8 * U, True))


TYPES = [("bf16", 128), ("i8", 128), ("f32", 128), ("bf16", 64), ("i8", 64), ("f32", 64)]


@pytest.mark.parametrize("kind,d", TYPES)
@pytest.mark.parametrize("bs,offs", [(16, [0, 3, 17, 0, 5, 0]), (24, [0, 23, 5, 1, 0, 2]), (1, [0] * 6)])
def test_few_rows(kind, d, bs, offs):
    """Up to four tokens a sequence (one 16-row tile), contexts from the new tokens alone to several steps."""
    su = Setup([4, 1, 3, 0, 4, 2], [4, 1, 33, 40, 128, 301], d=d, cache=kind, bs=bs, offs=offs)
    check(su, 2 * 4, masks_of(su))


@pytest.mark.parametrize("kind,d", TYPES)
@pytest.mark.parametrize("Hq,H", [(4, 4), (14, 2), (3, 1), (40, 2)])
def test_groups(kind, d, Hq, H):
    """Head groups of one, seven, three and twenty; trees of one to seventeen tokens."""
    su = Setup([1, 5, 17, 2, 12], [70, 5, 40, 131, 333], H=H, d=d, cache=kind, bs=16, offs=[1, 0, 7, 30, 0])
    check(su, Hq, masks_of(su, seed=Hq))


@pytest.mark.parametrize("kind,d", TYPES)
@pytest.mark.parametrize("window", [0, 40, 41, 64, 200])
def test_windows(kind, d, window):
    """Windows as long as the largest tree and longer; contexts shorter and longer than they are."""
    su = Setup([12, 40, 33, 3, 40], [100, 41, 170, 3, 260], H=2, d=d, cache=kind, bs=8, offs=[0, 2, 0, 0, 9])
    check(su, 4, masks_of(su, seed=window), window)


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
@pytest.mark.parametrize("q", [63, 64, 65, 130, 200])
@pytest.mark.parametrize("base", [0, 1, 63, 100])
def test_wide_trees(kind, q, base):
    """Trees of a word and more, that begin anywhere in a tile of keys; words to spare, and bits behind the last token."""
    su = Setup([q, 5], [base + q, base + 9], H=1, cache=kind, bs=16, offs=[0, 11])
    masks = masks_of(su, ["depth", "levels"], seed=q, words=q // 64 + 2)
    want = check(su, 4, masks)
    stray = masks.copy()
    for row, n in [(r, q) for r in range(q)] + [(q + r, 5) for r in range(5)]:
        for w in range(stray.shape[1]):
            keep = min(64, max(0, n - 64 * w))
            stray[row, w] |= np.uint64(((1 << 64) - 1) ^ ((1 << keep) - 1))
    got = kvc.kvc_attend_tree(su.cache(), su.step(), i64(stray), su.queries(4))
    assert torch.equal(got, want[0])
    got = kvc.kvc_attend_tree(su.cache(), su.step(), i64(stray), su.queries(4), window=max(q, 70))
    assert torch.equal(got, kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks), su.queries(4), window=max(q, 70)))


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
def test_any_masks(kind):
    """Masks that are no tree's: empty ones, tokens that do not see themselves, tokens that see later ones, with and without
    a context before them."""
    rng = np.random.default_rng(5)
    su = Setup([9, 70, 6], [9, 90, 300], H=2, cache=kind, bs=16)
    masks = rng.integers(0, 1 << 63, size=(su.N, 2), dtype=np.uint64) & rng.integers(0, 1 << 63, size=(su.N, 2), dtype=np.uint64)
    masks[[0, 3, 20, 80]] = 0
    check(su, 8, masks)
    check(su, 8, masks, window=75)


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
def test_contexts_shorter_than_the_new_tokens(kind):
    """Tokens without a place see nothing; the others see what has one."""
    su = Setup([20, 3, 70], [12, 0, 69], H=2, cache=kind, bs=16, offs=[3, 0, 0])
    check(su, 4, masks_of(su, ["chain", "levels", "depth"]))


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
def test_long_axis(kind):
    """Split ranges: a few rows and many over long contexts, one sequence and several."""
    su = Setup([8], [5003], H=2, cache=kind, bs=32)
    check(su, 8, masks_of(su, ["levels"]))
    su = Setup([60], [3001], H=1, cache=kind, offs=[5])
    check(su, 7, masks_of(su, ["depth"]))
    su = Setup([2, 16, 7], [2500, 4000, 17], H=1, cache=kind, offs=[40, 0, 0])
    check(su, 4, masks_of(su))
    check(su, 4, masks_of(su), window=1000)


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
def test_blocks_outside_the_pool(kind):
    su = Setup([8, 5], [100, 64], H=2, cache=kind, bs=16)
    su.tables[0, 2], su.tables[0, 6], su.tables[1, 3] = -1, su.nb, 1 << 30
    check(su, 4, masks_of(su))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("Hq", [2, 8, 32])
def test_no_numbers(kind, Hq):
    """What a token does not see has no effect, whatever its rows hold; what it sees counts."""
    su = Setup([8], [200], H=2, cache=kind, bs=16, paged=False)
    masks = masks_of(su, ["levels"])  # 0; 1 2 3; 4 5 6 (of 1), 7 (of 2)
    clean = kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks), su.queries(Hq))
    for kv in (0, 1):
        for bad in (float("nan"), float("inf"), -float("inf")):
            su.pools[kv, 0, 12, 192 + 5 - 192] = bad  # token 5's row
            got, _ = check(su, Hq, masks) if kv else (kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks), su.queries(Hq)), 0)
            others = [j for j in range(8) if j != 5]
            assert torch.equal(got[others], clean[others])
            assert not bool(torch.isfinite(got[5]).all())
            su.pools[kv, 0, 12, 5] = 0.5
            clean2 = kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks), su.queries(Hq))
            assert torch.equal(clean2[others], clean[others])


def test_scales_that_are_no_numbers():
    su = Setup([8], [200], H=2, cache="i8", bs=16, paged=False)
    masks = masks_of(su, ["levels"])
    for Hq in (2, 8):
        clean = kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks), su.queries(Hq))
        old = su.scales[:, 0, 12, 5].clone()
        for kv in (0, 1):
            su.scales[kv, 0, 12, 5] = float("nan")
            got = kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks), su.queries(Hq))
            others = [j for j in range(8) if j != 5]
            assert torch.equal(got[others], clean[others]) and bool(got[5].isnan().all())
            su.scales[:, 0, 12, 5] = old


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
def test_a_chain_is_causal(kind):
    """Masks of a chain, against the causal attention: to within twice the bounds of one."""
    su = Setup([30, 5], [100, 400], H=2, cache=kind)
    masks = masks_of(su, ["chain"])
    q = su.queries(8)
    out, lse = torch.empty_like(q), torch.empty(su.N, 8, device=DEV)
    kvc.kvc_attend(su.cache(), su.step(), q, out, lse=lse)
    compare(su, 8, masks, q, out, lse)
    check(su, 8, masks, q=q)


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
def test_views_scales_and_layers(kind):
    """Strided queries and results, head-major pools, a negative and a zero scale, the second layer."""
    su = Setup([6, 9], [60, 130], H=2, cache=kind, layers=2, head_major=True)
    masks = masks_of(su)
    wide = torch.randn(su.N, 8 + 4, su.d, generator=torch.Generator().manual_seed(3)).to(su.rows).to(DEV)
    q = wide[:, 2:10]
    for scale in (None, -0.2, 0.0):
        check(su, 8, masks, scale=scale, layer=1, q=q)
    want = kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks), q, layer=1)
    out = torch.full((8, su.N, su.d), 3.0, dtype=su.rows, device=DEV).transpose(0, 1)
    assert torch.equal(kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks), q, out, layer=1), want)


def test_rows_of_no_sequence_are_left():
    su = Setup([4, 3], [50, 60], H=2, cache="bf16")
    t = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    step = kvc.Step.on_device(t(1, 5, 8), t(50, 200), 9, 4, 100, torch.from_numpy(su.tables).to(torch.int32).to(DEV))
    q = torch.randn(9, 8, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    masks = np.concatenate([np.zeros((1, 1), np.uint64), masks_of(su), np.zeros((1, 1), np.uint64)])
    out, lse = torch.full_like(q, 5.0), torch.full((9, 8), 5.0, device=DEV)
    kvc.kvc_attend_tree(su.cache(), step, i64(masks), q, out, lse=lse)  # (the second's context passes the bound)
    left = [0, 5, 6, 7, 8]
    assert bool((out[left] == 5).all()) and bool((lse[left] == 5).all())
    want = kvc.kvc_attend_tree(su.cache(), kvc.Step([4], [50], step.tables[:1]), i64(masks[1:5]), q[1:5])
    assert torch.equal(out[1:5], want)


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
def test_captured(kind):
    """Replays follow masks, lengths and tables; eager calls between them use the same workspace."""
    su = Setup([16, 16], [700, 2000], H=2, cache=kind)
    cache, step, q = su.cache(), su.step(), su.queries(8)
    masks = i64(masks_of(su))
    ws = torch.empty(max(1, kvc.kvc_attend_workspace_bytes(cache, step, 8)), dtype=torch.uint8, device=DEV)
    out = kvc.kvc_attend_tree(cache, step, masks, q, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvc.kvc_attend_tree(cache, step, masks, q, out, workspace=ws)
    for s in range(4):
        new = masks_of(su, TREES[s:] + TREES[:s], seed=s)
        masks.copy_(i64(new))
        step.contexts.copy_(torch.tensor([700 - 31 * s, 2000 - 200 * s], dtype=torch.int32))
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, kvc.kvc_attend_tree(cache, step, masks, q, workspace=ws))
        su.ctx = [700 - 31 * s, 2000 - 200 * s]
        lse = torch.empty(su.N, 8, device=DEV)
        kvc.kvc_attend_tree(cache, step, masks, q, out, lse=lse, workspace=ws)
        compare(su, 8, new, q, out, lse)


def test_on_another_stream():
    su = Setup([8, 8], [700, 300], H=2)
    masks = i64(masks_of(su))
    want = kvc.kvc_attend_tree(su.cache(), su.step(), masks, su.queries(8))
    side = torch.cuda.Stream()
    step, q = su.step(), su.queries(8)
    side.wait_stream(torch.cuda.current_stream())
    out = kvc.kvc_attend_tree(su.cache(), step, masks, q, stream=side)
    side.synchronize()
    assert torch.equal(out, want)


def test_where_masks_are_on_the_host():
    su = Setup([8], [70], H=2)
    with pytest.raises(ValueError, match="one GPU"):
        kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks_of(su)).cpu(), su.queries(8))


@pytest.mark.parametrize("seed", range(6))
def test_drawn(seed):
    """Random lengths, groups, blocks, windows and trees."""
    rng = np.random.default_rng(100 + seed)
    for _ in range(4):
        n, kind = int(rng.integers(1, 5)), ["bf16", "i8", "f32"][int(rng.integers(0, 3))]
        new = [int(x) for x in np.exp(rng.uniform(0, np.log(90), size=n)).astype(int)]
        ctx = [q + int(x) for q, x in zip(new, np.exp(rng.uniform(0, np.log(900), size=n)).astype(int) - 1)]
        H, g, d = int(rng.integers(1, 4)), int(rng.integers(1, 9)), int(rng.choice([64, 128]))
        su = Setup(new, ctx, H=H, d=d, cache=kind, bs=int(rng.choice([1, 8, 16, 24, 64])),
                   offs=[int(x) for x in rng.integers(0, 50, size=n)], seed=seed)
        window = int(rng.choice([0, max(new) + int(rng.integers(0, 300))]))
        print(new, ctx, H, g, d, kind, window, flush=True)
        check(su, H * g, masks_of(su, seed=seed), window)


# Many sequences of different lengths: all their keys cut into equal runs (rows of 17-32 over int8 caches, and of 33-128),
# sequences and heads enough that a run is less than the longest sequence.  The last four, of 129-256 rows, have too few turns
# for the tallest tiles: they are worked on in ranges of 128-row tiles (test_attend_tree_tall_gpu.py has the tallest).
SHARES = [("i8", 128, 5, 8, 4), ("i8", 64, 3, 4, 7), ("bf16", 128, 9, 16, 4), ("i8", 128, 9, 16, 4), ("bf16", 64, 5, 9, 14),
          ("i8", 64, 17, 31, 4), ("bf16", 128, 30, 60, 4), ("i8", 128, 30, 60, 4), ("bf16", 64, 33, 64, 4), ("i8", 64, 33, 64, 4)]


def shares_setup(kind, d, lo, hi, seed=0, n=24):
    """Ragged contexts up to 1200; among them an empty one, new tokens alone, one shorter than its new tokens, and sequences
    without new tokens."""
    rng = np.random.default_rng(seed)
    new = rng.integers(lo, hi + 1, size=n)
    new[0] = hi
    ctx = new + np.exp(rng.uniform(0, np.log(1100), size=n)).astype(int)
    ctx[0], ctx[1], ctx[2], ctx[3] = 1200, 0, new[2], new[3] - 1
    new[4] = new[n - 1] = 0
    return Setup(new.tolist(), ctx.tolist(), H=2, d=d, cache=kind, bs=16, offs=rng.integers(0, 40, size=n).tolist(), seed=seed)


@pytest.mark.parametrize("kind,d,lo,hi,g", SHARES)
def test_shares(kind, d, lo, hi, g):
    su = shares_setup(kind, d, lo, hi)
    check(su, 2 * g, masks_of(su))


@pytest.mark.parametrize("kind,d,lo,hi,g", SHARES[::3])
def test_shares_windows_and_missing_blocks(kind, d, lo, hi, g):
    su = shares_setup(kind, d, lo, hi, seed=1)
    check(su, 2 * g, masks_of(su, seed=1), window=700)
    su.tables[0, 3], su.tables[0, 70], su.tables[6, 0] = -1, su.nb, 1 << 30
    check(su, 2 * g, masks_of(su, seed=1))


@pytest.mark.parametrize("kind,d,lo,hi,g", SHARES[1::3])
def test_shares_captured(kind, d, lo, hi, g):
    """Replays follow the lengths, on which the cuts depend; a second run over the same lengths gives the same bits."""
    su = shares_setup(kind, d, lo, hi, seed=2)
    cache, step, q = su.cache(), su.step(), su.queries(2 * g)
    masks = i64(masks_of(su))
    ws = torch.full((max(1, kvc.kvc_attend_workspace_bytes(cache, step, 2 * g)),), 255, dtype=torch.uint8, device=DEV)
    lse = torch.empty(su.N, 2 * g, device=DEV)
    out = torch.empty_like(q)
    kvc.kvc_attend_tree(cache, step, masks, q, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvc.kvc_attend_tree(cache, step, masks, q, out, lse=lse, workspace=ws)
    full = list(su.ctx)
    for s in range(3):
        su.ctx = [max(0, c - 97 * s * (i % 3)) for i, c in enumerate(full)]
        step.contexts.copy_(torch.tensor(su.ctx, dtype=torch.int32))
        out.fill_(9.0)
        lse.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        compare(su, 2 * g, masks.cpu().numpy(), q, out, lse)
        ws.fill_(255)
        assert torch.equal(out, kvc.kvc_attend_tree(cache, step, masks, q, workspace=ws))


@pytest.mark.parametrize("kind,d,lo,hi,g", [SHARES[2], SHARES[6]])
def test_shares_no_numbers(kind, d, lo, hi, g):
    """A value that is no number in a token's own row, and one in the context before it."""
    su = shares_setup(kind, d, lo, hi, seed=3)
    masks = masks_of(su, ["levels"], seed=3)
    p = su.offs[0] + su.ctx[0] - 1  # the first sequence's last token: a leaf
    su.pools[1, 0, su.tables[0, p // 16], p % 16] = float("nan")
    check(su, 2 * g, masks)
    p = su.offs[0] + 500
    su.pools[1, 0, su.tables[0, p // 16], p % 16, 0, 5] = float("inf")
    check(su, 2 * g, masks)


@pytest.mark.parametrize("kind,d,lo,hi,g", [SHARES[0], SHARES[2], SHARES[7]])
def test_shares_of_sequences_that_are_left_out(kind, d, lo, hi, g):
    """Sequences that contradict the bounds keep their rows, and the others get what they get without them."""
    su = shares_setup(kind, d, lo, hi, seed=4)
    q, masks = su.queries(2 * g), i64(masks_of(su, seed=4))
    step = su.step()
    want = kvc.kvc_attend_tree(su.cache(), step, masks, q)
    step.contexts[7], step.contexts[12] = 5000, -1
    out, lse = torch.full_like(q, 5.0), torch.full((su.N, 2 * g), 5.0, device=DEV)
    kvc.kvc_attend_tree(su.cache(), step, masks, q, out, lse=lse)
    starts = np.cumsum([0] + su.new)
    for i in range(len(su.new)):
        rows = slice(int(starts[i]), int(starts[i + 1]))
        if i in (7, 12):
            assert bool((out[rows] == 5).all()) and bool((lse[rows] == 5).all())
        else:  # (cut elsewhere: to within twice the roundings of one)
            a, b = out[rows].float(), want[rows].float()
            assert bool(((a - b).abs() <= 2.0 ** -6 * (b.abs() + b.abs().amax(-1, keepdim=True)) + 1e-6).all()) or not su.new[i]
