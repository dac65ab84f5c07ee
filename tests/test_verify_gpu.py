"""kvc_verify against the oracle: whole numbers, equal.  (Its sums in 64 bits end in another order than the oracle's: a
share that lies within 2^-50 of a border would decide otherwise, which no input here comes near but those that are exact.)"""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from paper_2609_34060_amd import kvc
from tests.draft_helpers import DEV, TREES, i32, tree

pytestmark = pytest.mark.gpu


class Drafts:
    """Trees with probabilities; tokens are drawn from their parent's draft row, or taken from its likeliest."""

    def __init__(self, parents, V, drawn, seed=0, noise=0.7, sharp=2.0, copies=False):
        g = torch.Generator().manual_seed(seed)
        self.parents, self.new, self.V = parents, [len(p) for p in parents], V
        self.N = sum(self.new)
        x = torch.randn(self.N, V, generator=g) * sharp
        self.target = torch.softmax(x, -1)
        y = torch.softmax(x + noise * torch.randn(self.N, V, generator=g), -1)
        self.draft = y if drawn else None
        self.tokens = torch.zeros(self.N, dtype=torch.int32)
        at = 0
        for p in parents:
            seen = {}
            for j in range(1, len(p)):
                if p[j] < 0:
                    continue
                row = y[at + p[j]]
                k = seen[p[j]] = seen.get(p[j], -1) + 1
                self.tokens[at + j] = int(torch.multinomial(row, 1, generator=g)) if drawn or copies else \
                    int(row.argsort(descending=True)[k % V])
            at += len(p)
        self.uniforms, self.last = torch.rand(self.N, generator=g), torch.rand(len(parents), generator=g)

    def step(self):
        return kvc.Step(self.new, [q + 3 for q in self.new], device=DEV)

    def run(self, children=0, step=None, **kw):
        dev = lambda t: None if t is None else t.to(DEV)
        path = torch.full((self.N,), 77, dtype=torch.int32, device=DEV)
        counts, chosen = (torch.full((len(self.new),), 77, dtype=torch.int32, device=DEV) for _ in range(2))
        return kvc.kvc_verify(self.step() if step is None else step, i32(np.concatenate(self.parents)), dev(self.tokens),
                              dev(self.target), dev(self.uniforms), dev(self.last), dev(self.draft), children, path=path,
                              counts=counts, chosen=chosen, **kw)

    def want(self, children=0):
        path, counts, chosen, at = [], [], [], 0
        for i, q in enumerate(self.new):
            if q == 0:
                counts.append(0)
                chosen.append(-1)
                continue
            s = slice(at, at + q)
            p, x = DO.verify(self.parents[i], self.tokens[s].numpy(), self.target[s].numpy(),
                             None if self.draft is None else self.draft[s].numpy(), self.uniforms[s].numpy(),
                             self.last[i], children)
            path += p + [-1] * (q - len(p))
            counts.append(len(p))
            chosen.append(x)
            at += q
        return path, counts, chosen

    def check(self, children=0, **kw):
        got, want = self.run(children, **kw), self.want(children)
        for g, w, what in zip(got, want, ("path", "counts", "chosen")):
            assert g.tolist() == list(w), what
        return want


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("V", [1, 2, 3, 5, 63, 257, 2047, 2048, 2049, 8193, 50021])
def test_vocabularies(drawn, V):
    rng = np.random.default_rng(V)
    trees = [tree(k, q, rng) for k, q in (("chain", 5), ("levels", 9), ("star", 3), ("depth", 7), ("chain", 1))]
    d = Drafts(trees, V, drawn, seed=V)
    for children in (0, 1, 2):
        d.check(children)


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("kind", ["chain", "levels", "depth", "star"])
@pytest.mark.parametrize("q", [2, 63, 64, 65, 200])
def test_trees(drawn, kind, q):
    """Trees of a wave's width and more, with drafts that are close to the target (long paths) and far from it."""
    rng = np.random.default_rng(q)
    for noise in (0.02, 3.0):
        d = Drafts([tree(kind, q, rng) for _ in range(4)], 300, drawn, seed=q, noise=noise, sharp=4.0)
        _, counts, _ = d.check()
        d.check(1)
        if kind == "chain" and drawn and noise < 0.1 and q > 60:
            assert max(counts) > 10


def test_the_largest_tree():
    d = Drafts([np.arange(-1, 1023), tree("levels", 1024, None), tree("star", 1024, None)], 50, True, noise=0.001)
    d.draft = d.target.clone()
    _, counts, _ = d.check()
    assert counts[0] == 1024  # (a draft that is the target is always accepted)
    d.draft = None
    d.check()


def test_many_sequences():
    rng = np.random.default_rng(9)
    sizes = rng.integers(0, 8, size=500)
    for drawn in (True, False):
        Drafts([tree(TREES[i % 4], int(q), rng) for i, q in enumerate(sizes)], 100, drawn, seed=3).check()


def test_siblings_of_one_token():
    """Drawn twice: tried again against what is left.  Chosen twice: the second is rejected."""
    for drawn in (True, False):
        for seed in range(8):
            d = Drafts([tree("star", 6, None), tree("levels", 13, None)], 4, drawn, seed=seed, sharp=0.3, copies=True)
            d.check()
    d = Drafts([tree("star", 4, None)], 4, False)
    d.tokens[:] = 2
    d.target[0] = torch.tensor([0.0, 0.0, 1.0, 0.0])
    d.uniforms[:] = 1.0
    assert d.check()[0] == [0, 1, -1, -1]
    d.target[0] = torch.tensor([0.5, 0.0, 0.5, 0.0])
    assert d.check()[0] == [0, -1, -1, -1] and d.check()[2] == [0]


@pytest.mark.parametrize("children", [0, 1])
def test_nothing_left(children):
    """A rejected token where nothing else is left either: the target's own probabilities; -1 where it has none."""
    d = Drafts([np.array([-1, 0]), np.array([-1, 0]), np.array([-1, 0])], 8, True)
    d.tokens[:] = 3
    d.target[:] = 0.125
    d.draft[:] = 0.125
    d.target[0, 3] = 0.0  # the first sequence's row: seven eighths, of which a half lies before token 4
    d.target[2] = 0.0     # the second's; the third accepts, whatever its number
    d.last[:] = 0.5
    assert d.check(children) == ([0, -1, 0, -1, 0, 1], [1, 1, 2], [4, -1, 4])
    d.target[:] = 0.0
    assert d.check(children)[2] == [-1, -1, -1]
    d.draft = None
    assert d.check(children)[2] == [-1, -1, -1]


def test_no_probabilities():
    """Negative ones, infinities and NaN count as 0, in either row; tokens outside the vocabulary have none."""
    rng = np.random.default_rng(1)
    for drawn in (True, False):
        for V in (40, 3000):
            d = Drafts([tree(k, 9, rng) for k in ("chain", "levels", "star", "depth")], V, drawn, seed=V)
            for x in (d.target,) + ((d.draft,) if drawn else ()):
                where = torch.rand(x.shape, generator=torch.Generator().manual_seed(5))
                x[where < 0.05] = float("nan")
                x[(where > 0.05) & (where < 0.1)] = float("inf")
                x[(where > 0.1) & (where < 0.15)] *= -1.0
                x[(where > 0.15) & (where < 0.2)] = -float("inf")
            for i, t in enumerate((-1, V, 2**31 - 1, -2**31)):
                d.tokens[5 + 9 * i] = t
            for children in (0, 1):
                d.check(children)


def test_random_numbers_at_their_ends():
    """0, the largest below 1, and what is none: 1, above, below and NaN."""
    rng = np.random.default_rng(2)
    for u in (0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, float("nan"), float("inf"), 2.0 ** -149):
        for drawn in (True, False):
            d = Drafts([tree(k, 6, rng) for k in ("chain", "levels")], 5000, drawn, seed=4)
            d.last[:] = u
            d.check()
            d.uniforms[:] = u
            for children in (0, 1):
                d.check(children)


def test_lines_that_end_nowhere():
    """A token whose parent is no earlier token is not accepted, nor are those behind it; a second root neither."""
    par = [np.array([-1, 1, 0, 5, -1, 4, 2, 99, -7, 6])]
    for drawn in (True, False):
        d = Drafts([np.where((par[0] >= 0) & (par[0] < np.arange(10)), par[0], 0)], 20, drawn, noise=0.01)
        d.parents = par
        d.uniforms[:] = 0.0
        want = d.check()
        assert set(want[0]) <= {0, 2, 6, 9, -1} and d.check(1)


def test_views_and_rows_of_no_sequence():
    """Rows of wider arrays, at any 4-byte place; sequences that contradict the bounds keep their rows of path."""
    rng = np.random.default_rng(6)
    for drawn in (True, False):
        d = Drafts([tree("levels", 6, rng), tree("chain", 4, rng), tree("chain", 3, rng)], 2053, drawn, seed=8)
        want = d.check()
        wide = lambda x: None if x is None else torch.nn.functional.pad(x, (3, 4))[:, 3:-4]
        d.target, d.draft = wide(d.target), wide(d.draft)
        buf = lambda x: None if x is None else torch.zeros(x.shape[0], 2061, device=DEV)[:, 3:2056].copy_(x)
        t, q = buf(d.target), buf(d.draft)
        got = kvc.kvc_verify(d.step(), i32(np.concatenate(d.parents)), d.tokens.to(DEV), t, d.uniforms.to(DEV),
                             d.last.to(DEV), q)
        assert [g.tolist() for g in got] == [list(w) for w in want]
        starts, ctx = i32([0, 6, 10, 13]), i32([9, 700, 9])  # the second's context passes the bound
        step = kvc.Step.on_device(starts, ctx, 13, 6, 20)
        path, counts, chosen = d.run(step=step)
        assert path.tolist() == want[0][:6] + [77] * 4 + want[0][10:]
        assert counts.tolist() == [want[1][0], 0, want[1][2]] and chosen.tolist() == [want[2][0], -1, want[2][2]]


def test_one_row_and_workspaces():
    d = Drafts([np.array([-1])], 100, True)
    assert d.check(children=1)[1] == [1]
    d = Drafts([np.arange(-1, 3)], 5000, True)
    need = kvc.kvc_verify_workspace_bytes(d.step(), 5000)
    d.check(workspace=torch.full((need,), 255, dtype=torch.uint8, device=DEV))
    with pytest.raises(kvc.KvcError):
        d.run(workspace=torch.empty(need - 1, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError, match="one GPU"):
        d.run(workspace=torch.empty(need, dtype=torch.uint8))


@pytest.mark.parametrize("drawn,children", [(True, 0), (True, 1), (False, 0)])
def test_distributed_as_the_target(drawn, children):
    """Over many sequences of one target, the first token after token 0 is distributed as the target's own, whatever the
    draft: each token's share lies within five standard deviations."""
    n, V, g = 20000, 7, torch.Generator().manual_seed(12)
    P = torch.softmax(torch.randn(V, generator=g) * 1.5, -1)
    Q = torch.softmax(torch.randn(V, generator=g) * 1.5, -1)
    par = i32([-1, 0, 0, 0] * n)
    tokens = torch.zeros(n, 4, dtype=torch.int32)
    if drawn:
        tokens[:, 1:] = torch.multinomial(Q, 3 * n, replacement=True, generator=g).view(n, 3).to(torch.int32)
    else:
        tokens[:, 1:] = torch.tensor([5, 2, 2], dtype=torch.int32)
    step = kvc.Step([4] * n, [9] * n, device=DEV)
    path, counts, chosen = kvc.kvc_verify(step, par, tokens.view(-1).to(DEV), P.repeat(4 * n, 1).to(DEV),
                                          torch.rand(4 * n, generator=g).to(DEV), torch.rand(n, generator=g).to(DEV),
                                          Q.repeat(4 * n, 1).to(DEV) if drawn else None, children)
    path, chosen = path.view(n, 4).cpu().long(), chosen.cpu().long()
    first = torch.where(counts.cpu() > 1, tokens.long().gather(1, path[:, 1:2].clamp(min=0))[:, 0], chosen)
    share = torch.bincount(first, minlength=V).double() / n
    p = P.double()
    assert bool(((share - p).abs() <= 5 * torch.sqrt(p * (1 - p) / n)).all())


@pytest.mark.parametrize("drawn,children", [(True, 0), (True, 1), (False, 0)])
def test_captured(drawn, children):
    """Replays follow all that the call reads; eager calls between them use the same workspace; another stream."""
    rng = np.random.default_rng(7)
    a = [Drafts([tree(k, 8, rng) for k in ("levels", "depth", "chain")], 4099, drawn, seed=s) for s in range(4)]
    dev = lambda t: None if t is None else t.to(DEV)
    d = a[0]
    step, par = d.step(), i32(np.concatenate(d.parents))
    state = [dev(x) for x in (d.tokens, d.target, d.uniforms, d.last)]
    draft = dev(d.draft)
    ws = torch.empty(kvc.kvc_verify_workspace_bytes(step, 4099), dtype=torch.uint8, device=DEV)
    out = kvc.kvc_verify(step, par, *state, draft, children, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvc.kvc_verify(step, par, *state, draft, children, *out, workspace=ws)
    side = torch.cuda.Stream()
    for b in a[1:] + a[:1]:
        par.copy_(i32(np.concatenate(b.parents)))
        for x, y in zip(state, (b.tokens, b.target, b.uniforms, b.last)):
            x.copy_(y)
        if drawn:
            draft.copy_(b.draft)
        for o in out:
            o.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        want = b.want(children)
        assert [o.tolist() for o in out] == [list(w) for w in want]
        b.check(children, workspace=ws)
        side.wait_stream(torch.cuda.current_stream())
        got = kvc.kvc_verify(step, par, *state, draft, children, stream=side)
        side.synchronize()
        assert [o.tolist() for o in got] == [list(w) for w in want]
