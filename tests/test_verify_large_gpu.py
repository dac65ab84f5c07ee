"""kvc_verify over vocabularies of more than 131072, whose sums are more than one to a lane: the same whole numbers as the
oracle's (see test_verify_gpu.py), wherever the next token lies."""
import numpy as np
import pytest
import torch

from tests.draft_helpers import tree
from tests.test_verify_gpu import Drafts

pytestmark = pytest.mark.gpu
PIECE, LANES = 2048, 64
MOST = 1.0 - 2.0 ** -24


def lanes(V):
    """Pieces of 2048 of a vocabulary, and how many of them a lane sums."""
    pieces = -(-V // PIECE)
    return pieces, -(-pieces // LANES)


VOCABS = [131072, 131073, 151936, 262144, 300001]


def test_sizes():
    assert [lanes(V)[1] for V in VOCABS] == [1, 2, 2, 2, 3]


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("V", VOCABS)
def test_next_tokens_everywhere(V, drawn):
    """Random numbers that end in the first, the middle and the last piece of a lane's, in the first and the last of all, at
    0 and at the largest below 1; one child tried and all of them."""
    pieces, run = lanes(V)
    places = [0, 1, run - 1, run, 2 * run - 1, 7 * run, 7 * run + run // 2, 7 * run + run - 1, pieces // 2, pieces - 2, pieces - 1]
    numbers = [0.0, MOST] + [(p + 0.4) / pieces for p in places]
    d = Drafts([tree("star", 3, None) for _ in numbers], V, drawn, seed=V, sharp=0.3, noise=0.3)
    d.last = torch.tensor(numbers, dtype=torch.float32)
    for children in (0, 1):
        _, _, chosen = d.check(children)
    d.uniforms[:] = MOST  # (nearly all are rejected: the token after token 0, from what is left)
    for children in (0, 1):
        _, counts, chosen = d.check(children)
    assert counts.count(1) > len(numbers) // 3
    assert len({x // PIECE for x in chosen}) > len(places) // 2


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("V", VOCABS[1:])
def test_what_is_left_in_one_piece(V, drawn):
    """What is left lies in a single piece, or in two of one lane: the first, a middle or the last of a lane's, the last of
    all; a few of its tokens, so that shares end at them and behind the last."""
    pieces, run = lanes(V)
    where = [(0,), (1,), (run - 1,), (3 * run,), (3 * run + run - 1,), (4 * run, 4 * run + run - 1), (pieces - 1,),
             (pieces - 2, pieces - 1), (0, pieces - 1)]
    d = Drafts([np.array([-1, 0])] * (3 * len(where)), V, drawn, seed=1)
    g = torch.Generator().manual_seed(V)
    d.target.zero_()
    for i in range(3 * len(where)):
        row = d.target[2 * i]
        for p in where[i % len(where)]:
            n = min(PIECE, V - p * PIECE)
            at = p * PIECE + torch.randint(0, n, (5,), generator=g)
            row[at] = torch.rand(5, generator=g) + 0.05
            row[p * PIECE + (n - 1 if i % 2 else 0)] = 0.1
        row /= 2.0 * row.sum()
        row[99] = 0.5  # the child's, which what is left does not have
        d.tokens[2 * i + 1] = 99
    if drawn:
        d.draft.zero_()
        d.draft[:, 99] = 1.0
    d.uniforms[:] = MOST
    d.last = torch.tensor([[0.0, 0.5, MOST][i // len(where)] for i in range(3 * len(where))], dtype=torch.float32)
    for children in (0, 1):
        _, counts, chosen = d.check(children)
        assert set(counts) == {1}
        for i, x in enumerate(chosen):
            assert x // PIECE in where[i % len(where)] and x != 99


@pytest.mark.parametrize("V", VOCABS)
def test_trees_of_drawn_tokens(V):
    """Rounds over the whole row for second and later children; nothing left, and rows without anything."""
    rng = np.random.default_rng(V)
    d = Drafts([tree("levels", 7, rng), tree("star", 5, rng), tree("chain", 3, rng), tree("star", 4, rng)], V, True, seed=2)
    d.check()
    d.draft[7:12] = d.target[7:12]  # the star's draft is its target: its first child is accepted
    d.target[15:] = 0.0             # the last one's has nothing
    want = d.check()
    assert want[1][1] == 2 and want[1][3] == 1 and want[2][3] == -1
    d.uniforms[:] = MOST
    d.draft[15:] = d.draft[15].clone()
    d.target[15:] = d.draft[15:] * 0.25
    d.check()  # (a quarter of the draft's: nothing left after the first child; the target's own)
