"""kvc_keep: rows moved bit for bit, everything else as it was."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from oracle import serve_oracle as SO
from paper_2609_34060_amd import kvc
from tests.draft_helpers import DEV, i32
from tests.test_serve_gpu import Setup

pytestmark = pytest.mark.gpu


def check(su, paths, counts=None, layers=None, stream=None):
    counts = [len(p) for p in paths] if counts is None else counts
    path = np.full(su.N, -1, dtype=np.int64)
    want = su.pools.cpu().clone()
    scales = None if su.scales is None else su.scales.cpu().clone()
    lb, le = (0, su.layers) if layers is None else layers
    at = 0
    for i, (p, q) in enumerate(zip(paths, su.new)):
        path[at:at + len(p)] = p
        full = [int(x) for x in path[at:at + q]]
        base = su.ctx[i] - q
        moved = []
        for a, b in DO.keep(full, counts[i], q):
            come, to = (SO.place(base + x, su.offs[i], su.bs, su.nb, None if su.tables is None else su.tables[i]) for x in (a, b))
            if come is not None and to is not None:
                moved.append((come, to, want[:, lb:le, come[0], come[1]].clone(),
                              None if scales is None else scales[:, lb:le, come[0], come[1]].clone()))
        for come, to, row, sc in moved:
            want[:, lb:le, to[0], to[1]] = row
            if sc is not None:
                scales[:, lb:le, to[0], to[1]] = sc
        at += q
    kvc.kvc_keep(su.cache(), su.step(), i32(path), i32(counts), lb, le, stream=stream)
    torch.cuda.synchronize()
    bits = {torch.bfloat16: torch.int16, torch.float32: torch.int32, torch.int8: torch.int8}[want.dtype]
    assert torch.equal(su.pools.cpu().view(bits), want.view(bits))
    if scales is not None:
        assert torch.equal(su.scales.cpu(), scales)


KINDS = ["bf16", "i8", "f32"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bs", [1, 8, 16, 24])
def test_paths(kind, d, bs):
    """Nothing accepted but token 0, whole chains, paths with gaps; tokens that come from where others go."""
    su = Setup([8, 5, 12, 1, 9, 0, 30], [100, 5, 40, 7, 300, 20, 64], H=3, d=d, cache=kind, bs=bs,
               offs=[0, 3, 0, 17, 5, 0, 2], layers=3)
    check(su, [[0, 2, 3, 4, 5], [0, 1, 2, 3, 4], [0, 5, 11], [0], [0, 1, 3, 4, 8], [], [0, 2, 4, 6, 8, 10, 12, 14, 16, 18, 29]])


@pytest.mark.parametrize("kind", KINDS)
def test_long_paths(kind):
    """Hundreds of tokens, each of which goes where one before it came from."""
    su = Setup([300, 200], [310, 200], H=1, cache=kind, layers=2)
    check(su, [list(range(1, 300)), sorted(np.random.default_rng(0).permutation(200)[:130].tolist())])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H", [1, 2, 8, 33])
def test_heads_and_layouts(kind, H):
    """Rows of less than a wave and of several; pools with a head's tokens next to one another."""
    for head_major in (False, True):
        su = Setup([7, 7], [20, 33], H=H, cache=kind, layers=2, head_major=head_major)
        check(su, [[0, 3, 6], [0, 2, 3, 5]])


@pytest.mark.parametrize("kind", ["bf16", "i8"])
def test_many_layers(kind):
    """More layers than one launch takes, and a range of them."""
    for layers in (None, (3, 5), (60, 70), (7, 7)):
        su = Setup([6, 4], [20, 9], H=2, d=64, cache=kind, layers=70)
        check(su, [[0, 2, 5], [0, 3]], layers=layers)


def test_paths_that_end_early():
    """A path ends before the first token that does not ascend or is none of the sequence's; counts beyond the tokens and
    below 0."""
    su = Setup([8] * 7, [20] * 7, H=2)
    check(su, [[0, 2, 2, 4], [0, 3, 1, 6], [0, 2, 8], [-1, 3, 4], [1, 4, 7], [0, 2, 4], [0, 2**31 - 1]],
          [4, 4, 3, 3, 100, -5, 2])


def test_tokens_without_a_place():
    """Contexts shorter than the new tokens, and blocks outside the pool."""
    su = Setup([10, 10, 6], [6, 0, 90], H=2, bs=4)
    su.tables[2, 21], su.tables[2, 22] = -1, su.nb
    check(su, [[2, 3, 5, 6, 8, 9], [0, 3], [0, 2, 4, 5]])


def test_sequences_that_are_left_out():
    su = Setup([4, 4], [20, 20], H=2)
    before = su.pools.clone()
    step = kvc.Step.on_device(i32([0, 4, 8]), i32([200, 2000]), 8, 4, 100, torch.from_numpy(su.tables).to(torch.int32).to(DEV))
    kvc.kvc_keep(su.cache(), step, i32([0, 2, 3, -1] * 2), i32([3, 3]))
    assert torch.equal(su.pools, before)


def test_captured_and_on_another_stream():
    """Replays follow paths, counts and lengths."""
    su = Setup([8, 8], [40, 50], H=2, layers=2)
    twin = Setup([8, 8], [40, 50], H=2, layers=2)
    cache, step = su.cache(), su.step()
    path, counts = i32([0, 1] + [-1] * 6 + [0] + [-1] * 7), i32([2, 1])
    kvc.kvc_keep(cache, step, path, counts)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvc.kvc_keep(cache, step, path, counts)
    for s, p in enumerate(([0, 2, 3, 7], [1, 5], [0, 1, 2, 4, 6])):
        path[:len(p)] = i32(p)
        path[8:8 + len(p)] = i32(p)
        counts.copy_(i32([len(p), len(p)]))
        step.contexts.copy_(i32([40 - s, 50 - s]))
        graph.replay()
        torch.cuda.synchronize()
        twin.ctx = [40 - s, 50 - s]
        side = torch.cuda.Stream()
        check(twin, [p, p], stream=side)
        assert torch.equal(su.pools, twin.pools)
