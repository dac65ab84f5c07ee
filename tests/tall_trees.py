"""Steps of drafted tokens whose lists of rows reach the tallest tiles, and the plan that the library makes for them."""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Tuple

import numpy as np

from paper_2609_34060_amd import kvc


class Tall(NamedTuple):
    """`seqs` sequences of up to `most` new tokens, `group` heads on each of `heads`, contexts up to `ctx`."""
    kind: str
    dim: int
    seqs: int
    least: int
    most: int
    heads: int
    group: int
    ctx: int
    route: Tuple[int, bool, bool]  # rows of a tile, whether a list is one tile, whether the keys are shared out


# Lists of 129-256 rows over many sequences, whose keys are cut into equal runs; the same over one sequence; lists of more
# than a tile.  Each type and head dimension, with as many turns of 64 keys in all as the tallest tiles begin at.
TALL = [
    Tall("bf16", 128, 24, 33, 64, 4, 4, 1400, (256, True, True)),
    Tall("i8", 128, 24, 33, 64, 4, 4, 1400, (256, True, True)),
    Tall("bf16", 64, 26, 19, 36, 4, 7, 1400, (256, True, True)),
    Tall("i8", 64, 26, 19, 36, 4, 7, 1400, (256, True, True)),
    Tall("bf16", 128, 1, 64, 64, 8, 4, 16100, (256, True, False)),
    Tall("i8", 128, 1, 64, 64, 8, 4, 12100, (256, True, False)),
    Tall("bf16", 64, 1, 33, 33, 8, 4, 16077, (256, True, False)),
    Tall("i8", 64, 1, 33, 33, 8, 4, 12161, (256, True, False)),
    Tall("bf16", 128, 1, 60, 60, 4, 7, 16200, (256, False, False)),
    Tall("i8", 128, 1, 60, 60, 4, 7, 12200, (256, False, False)),
    Tall("bf16", 64, 3, 65, 100, 4, 4, 6500, (256, False, False)),
    Tall("i8", 64, 3, 65, 100, 4, 4, 4600, (256, False, False)),
]
# The same kinds of steps under 128-row tiles: a list a tile, shared out or not, and lists of more than a tile.
LOW = [
    Tall("bf16", 128, 24, 9, 32, 2, 4, 1200, (128, True, True)),
    Tall("i8", 64, 24, 9, 32, 2, 4, 1200, (128, True, True)),
    Tall("bf16", 64, 1, 30, 30, 2, 4, 1500, (128, True, False)),
    Tall("i8", 128, 1, 30, 30, 2, 4, 1500, (128, True, False)),
    Tall("bf16", 128, 24, 30, 60, 2, 4, 1200, (128, False, False)),
    Tall("i8", 128, 24, 30, 60, 2, 4, 1200, (128, False, False)),
]


def lengths(t: Tall, seed: int = 0):
    """New tokens and contexts; of many sequences, an empty one, new tokens alone, one shorter than its new tokens, and
    sequences without new tokens among them."""
    rng = np.random.default_rng(seed)
    new = rng.integers(t.least, t.most + 1, size=t.seqs)
    new[0] = t.most
    ctx = new + np.exp(rng.uniform(0, np.log(t.ctx - t.most), size=t.seqs)).astype(int)
    ctx[0] = t.ctx
    if t.seqs > 8:
        ctx[1], ctx[2], ctx[3], ctx[5] = 0, new[2], new[3] - 1, t.ctx - 1
        new[4] = new[t.seqs - 1] = 0
    return new.tolist(), ctx.tolist()


class _Plan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tile_rows", "direct", "tiles", "splits", "chunk", "shared")] + \
        [(n, ctypes.c_size_t) for n in ("bytes", "most_bytes")]


def plan(kind: str, seqs: int, rows: int, max_new: int, span: int, context: int, heads: int, group: int, dim: int,
         tree: bool = True) -> _Plan:
    """kvc::plan_attend, on the host."""
    call = kvc.load()._ZN3kvc11plan_attendE9kvc_dtypeiiilliiib
    call.restype = _Plan
    call.argtypes = [ctypes.c_int] * 4 + [ctypes.c_long] * 2 + [ctypes.c_int] * 3 + [ctypes.c_bool]
    return call({"f32": kvc.KVC_F32, "bf16": kvc.KVC_BF16, "i8": kvc.KVC_I8}[kind], seqs, rows, max_new, span, context, heads,
                group, dim, tree)


def route(t: Tall, window: int = 0, seed: int = 0) -> Tuple[int, bool, bool]:
    new, ctx = lengths(t, seed)
    span = min(max(ctx), window + max(new)) if window else max(ctx)
    p = plan(t.kind, t.seqs, sum(new), max(new), span, max(ctx), t.heads, t.group, t.dim)
    return p.tile_rows, bool(p.direct), p.shared > 0


SEEDS = 4  # of the lengths that the tests draw


def window_of(t: Tall) -> int:
    """A window that hides a part of the longest contexts and leaves the plan as it is."""
    return t.ctx - 150
