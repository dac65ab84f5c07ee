"""kvc_tree against the oracle: whole numbers, equal."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from paper_2609_34060_amd import kvc
from tests.draft_helpers import DEV, TREES, i32, tree

pytestmark = pytest.mark.gpu


def check(parents, ctx, words=None, step=None):
    """parents: a list of arrays, one a sequence."""
    new = [len(p) for p in parents]
    words = max(1, -(-max(new) // 64)) if words is None else words
    step = kvc.Step(new, ctx, device=DEV) if step is None else step
    masks = torch.full((sum(new), words), 77, dtype=torch.int64, device=DEV)
    positions = torch.full((sum(new),), 77, dtype=torch.int32, device=DEV)
    got = kvc.kvc_tree(step, i32(np.concatenate(parents)), masks, positions)
    assert got[0] is masks and got[1] is positions
    want = [DO.tree(p, c - len(p), words) for p, c in zip(parents, ctx)]
    assert np.array_equal(masks.cpu().numpy().view(np.uint64), np.concatenate([w[0] for w in want]))
    assert np.array_equal(positions.cpu().numpy(), np.concatenate([w[1] for w in want]))


@pytest.mark.parametrize("kind", TREES)
@pytest.mark.parametrize("q", [1, 2, 63, 64, 65, 127, 129, 257, 1000, 1024])
def test_shapes(kind, q):
    check([tree(kind, q, np.random.default_rng(q))], [q + 5])


@pytest.mark.parametrize("words", [2, 3, 16, 40])
def test_more_words_than_needed(words):
    rng = np.random.default_rng(words)
    check([tree(k, 100 + i, rng) for i, k in enumerate(TREES)], [200] * 5, words)


def test_batches():
    """Ragged sequences, some without tokens, contexts shorter than the new tokens (their positions lie below 0)."""
    rng = np.random.default_rng(3)
    sizes = [5, 0, 300, 1, 64, 0, 17, 128, 2]
    trees = [tree(TREES[i % 5], q, rng) for i, q in enumerate(sizes)]
    check(trees, [int(rng.integers(0, 400)) for _ in sizes])
    sizes = rng.integers(0, 70, size=700)
    check([tree(TREES[i % 5], int(q), rng) for i, q in enumerate(sizes)], [100] * 700)


def test_lines_that_end_nowhere():
    """Parents that are no earlier token, and those who descend from such a token: empty masks and position -1."""
    par = np.array([-1, 0, 2, 1, 7, 3, -2, 6, 0, 99, 9, 2**31 - 1, -2**31, 12, 11, 8])
    check([par, tree("chain", 70, None), np.array([0, -1, 1, 0])], [40, 100, 4])
    par = np.arange(-1, 199)
    par[100] = 150
    check([par], [1000])


def test_rows_of_no_sequence_are_left():
    """Rows behind the last sequence, and those of sequences that contradict the bounds."""
    starts, ctx = i32([2, 5, 4, 9]), i32([10, 10, 10])
    step = kvc.Step.on_device(starts, ctx, 12, 4, 20)  # the second is longer than it may be long: it descends; the third has five
    masks = torch.full((12, 1), 77, dtype=torch.int64, device=DEV)
    positions = torch.full((12,), 77, dtype=torch.int32, device=DEV)
    kvc.kvc_tree(step, i32([-1, -1, -1, 0, 1] + [-1] * 7), masks, positions)
    assert masks[:, 0].tolist() == [77, 77, 1, 3, 7] + [77] * 7
    assert positions.tolist() == [77, 77, 7, 8, 9] + [77] * 7


def test_without_positions():
    step = kvc.Step([3], [10], device=DEV)
    parents, masks = i32([-1, 0, 0]), torch.zeros(3, 1, dtype=torch.int64, device=DEV)
    st = kvc.load().kvc_tree(step._at, parents.data_ptr(), masks.data_ptr(), 1, None, torch.cuda.current_stream().cuda_stream)
    assert st == 0 and masks[:, 0].tolist() == [1, 3, 5]


def test_captured():
    """Replays follow parents and lengths."""
    rng = np.random.default_rng(11)
    starts, ctx = i32([0, 40, 80]), i32([50, 60])
    step = kvc.Step.on_device(starts, ctx, 80, 80, 100)
    parents = i32(np.concatenate([tree("levels", 40, rng)] * 2))
    masks, positions = kvc.kvc_tree(step, parents)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvc.kvc_tree(step, parents, masks, positions)
    for kind, cut in (("depth", 13), ("forest", 40), ("star", 1), ("chain", 79)):
        trees = [tree(kind, cut, rng), tree(kind, 80 - cut, rng)]
        starts.copy_(i32([0, cut, 80]))
        parents.copy_(i32(np.concatenate(trees)))
        masks.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        want = [DO.tree(p, c - len(p), 2) for p, c in zip(trees, (50, 60))]
        assert np.array_equal(masks.cpu().numpy().view(np.uint64), np.concatenate([w[0] for w in want]))
        assert np.array_equal(positions.cpu().numpy(), np.concatenate([w[1] for w in want]))
