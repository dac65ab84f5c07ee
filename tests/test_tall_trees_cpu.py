"""The plans behind the tests of tall trees: each step is worked on by the kernel that its test is for."""
import pytest

from tests.tall_trees import LOW, SEEDS, TALL, route, window_of


@pytest.mark.parametrize("t", TALL + LOW)
def test_routes(t):
    for seed in range(SEEDS):
        assert route(t, seed=seed) == t.route


@pytest.mark.parametrize("t", TALL)
def test_routes_under_a_window(t):
    assert route(t, window_of(t), seed=1) == t.route


def test_every_tall_kernel_is_reached():
    """256 rows a tile: both types, both head dimensions, with and without shares, lists of one tile and of more."""
    reached = {(t.kind, t.dim, *t.route[1:]) for t in TALL}
    assert reached == {(k, d, direct, shared) for k in ("bf16", "i8") for d in (64, 128)
                       for direct, shared in ((True, True), (True, False), (False, False))}
