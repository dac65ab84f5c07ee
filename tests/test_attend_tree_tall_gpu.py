"""kvc_attend_tree where there are many rows: lists of more than 128 rows in the tallest tiles, one tile a list and several,
with the keys shared out and in ranges, against float64 on the GPU.  test_tall_trees_cpu.py holds the plans to these kernels.

Bounds as in test_attend_tree_gpu.py, with u = 2^-24 and A the weighted mean of |v|: a score is off by e = (d + 4) u mass +
4 u |s|, a weight by a factor of 1 + 2 e + 8 u, sums over n weights by n u; so the quotient by (4 e + 16 u + 2 n u) A; 2^-8 A
of a weight's rounding to bfloat16, 2^-8 |out| of the result's.  lse is off by 2 e + n u + 8 u |lse| + 8 u."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from paper_2609_34060_amd import kvc
from tests.draft_helpers import DEV, TREES, i64, tree
from tests.tall_trees import LOW, TALL, lengths, route, window_of
from tests.test_serve_gpu import U, Setup

pytestmark = pytest.mark.gpu


def setup(t, seed=0):
    new, ctx = lengths(t, seed)
    offs = np.random.default_rng(seed + 9).integers(0, 40, size=t.seqs).tolist()
    return Setup(new, ctx, H=t.heads, d=t.dim, cache=t.kind, bs=16, offs=offs, seed=seed)


def masks_of(su, kinds=TREES, seed=0):
    rng, words = np.random.default_rng(seed), -(-max(su.new) // 64)
    return np.concatenate([DO.tree(tree(kinds[i % len(kinds)], q, rng), 0, words)[0] for i, q in enumerate(su.new)])


def reference(su, q, masks, window=0):
    """out, its bound, lse and its bound, in float64."""
    k, v = (su.pools[j, 0].double() for j in range(2))
    if su.scales is not None:
        k, v = (x * su.scales[j, 0].double()[..., None] for j, x in enumerate((k, v)))
    Hq, g = q.shape[1], q.shape[1] // su.H
    out, bound = (torch.zeros(su.N, Hq, su.d, dtype=torch.float64, device=DEV) for _ in range(2))
    lse, lbound = (torch.zeros(su.N, Hq, dtype=torch.float64, device=DEV) for _ in range(2))
    at = 0
    for i, (n, c) in enumerate(zip(su.new, su.ctx)):
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        base, t = c - n, torch.arange(c, device=DEV)
        place = su.offs[i] + t
        blk = torch.from_numpy(su.tables[i]).to(DEV)[place // su.bs]
        there = (blk >= 0) & (blk < su.nb)
        slot, blk = place % su.bs, torch.where(there, blk, 0)
        bits = torch.from_numpy(DO.bits(masks[rows], n)).to(DEV)
        pos = base - 1 + bits.sum(1)
        see = torch.zeros(n, c, dtype=torch.bool, device=DEV)
        if base > 0:
            see[:, :base] = (t[None, :base] > pos[:, None] - window) if window else True
        see[:, max(0, base):] = bits[:, max(0, -base):]
        see &= there[None]
        see[:max(0, -base)] = False  # (tokens without a place)
        if c == 0:
            lse[rows] = -torch.inf
            continue
        for h in range(su.H):
            kh, vh = k[blk, slot, h], v[blk, slot, h]
            for j in range(h * g, (h + 1) * g):
                x = q[rows, j].double()
                s = (x @ kh.t().contiguous()) * su.d ** -0.5
                mass = (x.abs() @ kh.abs().t().contiguous()) * su.d ** -0.5
                s = torch.where(see, s, -torch.inf)
                e = (su.d + 4) * U * torch.where(see, mass, 0).amax(-1) + 4 * U * torch.where(see, s.abs(), 0).amax(-1)
                m = s.amax(-1, keepdim=True).clamp(min=-1e300)
                p = torch.exp(s - m)
                total = p.sum(-1, keepdim=True)
                p = p / total.clamp(min=1e-300)
                o, mean = p @ vh, p @ vh.abs()
                out[rows, j] = o
                bound[rows, j] = (4 * e + (16 + 2 * c) * U + 2.0 ** -8)[:, None] * mean + 2.0 ** -8 * o.abs() + 1e-30
                lse[rows, j] = (m + total.log())[:, 0]
                lbound[rows, j] = 2 * e + (c + 8) * U + 8 * U * lse[rows, j].abs()
    return out, bound, lse, lbound


def compare(su, q, masks, got, lse, window=0):
    out, bound, rlse, lbound = reference(su, q, masks, window)
    none = rlse == -torch.inf
    assert torch.equal(none, lse == -torch.inf) and not bool(got[none].any())
    err = (got.double() - out).abs()
    assert bool((err <= bound).all()), float((err / bound).max())
    assert bool(((lse.double() - rlse).abs()[~none] <= lbound[~none]).all())


def check(su, t, masks, window=0):
    q = su.queries(t.heads * t.group)
    lse = torch.full((su.N, t.heads * t.group), 77.0, device=DEV)
    got = torch.full_like(q, 77.0)
    kvc.kvc_attend_tree(su.cache(), su.step(), i64(masks), q, got, lse=lse, window=window)
    compare(su, q, masks, got, lse, window)
    return got


@pytest.mark.parametrize("t", TALL + LOW)
def test_trees(t):
    assert route(t) == t.route
    su = setup(t)
    check(su, t, masks_of(su, TREES if t.seqs > 1 else ["depth"]))


@pytest.mark.parametrize("t", TALL)
def test_windows_and_missing_blocks(t):
    """A window that ends within the longest contexts; blocks that are not there: at a context's start, within it and among
    the new tokens."""
    assert route(t, window_of(t), seed=1) == t.route
    su = setup(t, 1)
    masks = masks_of(su, seed=1)
    check(su, t, masks, window_of(t))
    last = (su.offs[0] + su.ctx[0] - 3) // 16
    su.tables[0, 3], su.tables[0, 70], su.tables[0, last], su.tables[t.seqs - 1, 0] = -1, su.nb, 1 << 30, -1
    check(su, t, masks)
    check(su, t, masks, window_of(t))


@pytest.mark.parametrize("t", TALL)
def test_any_masks(t):
    """Masks that are no tree's: empty ones, tokens that do not see themselves, tokens that see later ones."""
    su = setup(t, 2)
    rng, words = np.random.default_rng(5), -(-max(su.new) // 64)
    draw = lambda: rng.integers(0, 1 << 63, size=(su.N, words), dtype=np.uint64)
    masks = draw() & draw()
    masks[::7] = 0
    check(su, t, masks)


@pytest.mark.parametrize("t", TALL)
def test_captured(t):
    """Replays follow lengths and masks, eager calls between them use the same workspace, and the same call gives the same
    bits whatever the workspace held."""
    su = setup(t, 3)
    Hq = t.heads * t.group
    cache, step, q = su.cache(), su.step(), su.queries(Hq)
    masks = i64(masks_of(su, seed=3))
    ws = torch.full((max(1, kvc.kvc_attend_workspace_bytes(cache, step, Hq)),), 255, dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(q), torch.empty(su.N, Hq, device=DEV)
    kvc.kvc_attend_tree(cache, step, masks, q, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvc.kvc_attend_tree(cache, step, masks, q, out, lse=lse, workspace=ws)
    full = list(su.ctx)
    for s in range(3):
        new = masks_of(su, TREES[s:] + TREES[:s], seed=s)
        masks.copy_(i64(new))
        su.ctx = [max(0, c - 197 * s * (1 + i % 3)) for i, c in enumerate(full)]
        step.contexts.copy_(torch.tensor(su.ctx, dtype=torch.int32))
        out.fill_(9.0)
        lse.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        compare(su, q, new, out, lse)
        ws.fill_(255)
        assert torch.equal(out, kvc.kvc_attend_tree(cache, step, masks, q, workspace=ws))


@pytest.mark.parametrize("t", TALL)
def test_no_numbers_where_nothing_looks(t):
    """NaN and infinities (of an 8-bit cache: scales) past the contexts, before every window, and in the rows of new tokens
    that no other token sees (a star's leaves) reach nothing but those tokens themselves, bit for bit."""
    su = setup(t, 2)
    masks = i64(masks_of(su, ["star"]))
    Hq, window = t.heads * t.group, window_of(t)
    q, cache, step = su.queries(Hq), su.cache(), su.step()
    clean = kvc.kvc_attend_tree(cache, step, masks, q, window=window)
    assert bool(torch.isfinite(clean).all())
    dirty = torch.zeros(su.N, dtype=torch.bool)
    at = 0
    for i, (n, c) in enumerate(zip(su.new, su.ctx)):
        base, own = c - n, [j for j in range(1, n, 5) if c - n + j >= 0]
        hidden = list(range(0, max(0, base - window), 7))
        for e, p in enumerate(hidden + [base + j for j in own] + [c]):
            b, s = (su.offs[i] + p) // 16, (su.offs[i] + p) % 16
            b = su.tables[i][b] if b < su.tables.shape[1] else -1
            if b < 0:
                continue
            bad = [float("nan"), float("inf"), -float("inf")][e % 3]
            if t.kind == "i8":
                su.scales[1, 0, b, s] = bad
            else:
                su.pools[1, 0, b, s] = bad
        dirty[[at + j for j in own]] = True
        at += n
    got = kvc.kvc_attend_tree(cache, step, masks, q, window=window)
    assert torch.equal(got[~dirty.to(DEV)], clean[~dirty.to(DEV)])
    assert not bool(torch.isfinite(got[dirty.to(DEV)]).all(-1).any())


@pytest.mark.parametrize("t", [t for t in TALL if t.kind == "bf16"])
def test_a_value_that_all_see(t):
    """An infinity in a context shows in its feature, in every row that has it before it and its KV head, and nowhere else."""
    su = setup(t, 3)
    masks, Hq = i64(masks_of(su, seed=3)), t.heads * t.group
    q, cache, step = su.queries(Hq), su.cache(), su.step()
    clean = kvc.kvc_attend_tree(cache, step, masks, q)
    assert bool(torch.isfinite(clean).all())
    p = su.offs[0] + 500
    su.pools[1, 0, su.tables[0, p // 16], p % 16, 1, 5] = float("inf")
    got = kvc.kvc_attend_tree(cache, step, masks, q)
    rows = got[:su.new[0], t.group:2 * t.group, 5]
    assert bool((rows == float("inf")).all())
    rows.copy_(clean[:su.new[0], t.group:2 * t.group, 5])
    assert torch.equal(got, clean)


@pytest.mark.parametrize("t", [t for t in TALL if t.route[2]])
def test_sequences_that_are_left_out(t):
    """Sequences that contradict the bounds keep their rows; the others are as right as without them."""
    su = setup(t, 3)
    Hq = t.heads * t.group
    q, masks, step = su.queries(Hq), masks_of(su, seed=4), su.step()
    step.contexts[7], step.contexts[12] = t.ctx + 1, -1
    out, lse = torch.full_like(q, 5.0), torch.full((su.N, Hq), 5.0, device=DEV)
    kvc.kvc_attend_tree(su.cache(), step, i64(masks), q, out, lse=lse)
    starts = np.cumsum([0] + su.new)
    left = torch.zeros(su.N, dtype=torch.bool, device=DEV)
    for i in (7, 12):
        left[int(starts[i]):int(starts[i + 1])] = True
    assert bool((out[left] == 5).all()) and bool((lse[left] == 5).all())
    want, bound, rlse, lbound = reference(su, q, masks)
    assert bool(((out.double() - want).abs() <= bound)[~left].all())
    some = ~left[:, None] & (rlse > -torch.inf)
    assert bool(((lse.double() - rlse).abs() <= lbound)[some].all())
