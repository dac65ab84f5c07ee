"""A served step in float64, written from the definitions (test infrastructure only).

Sequence i of a step has q new tokens, the last of its c context tokens; context token t sits at position off + t of its
blocks.  A place is (block, slot), or None where the token has none: a negative context index, or a block id outside the
pool."""
from __future__ import annotations

import math
from typing import List, Optional, Sequence, Tuple

import numpy as np


def place(t: int, off: int, block_size: int, num_blocks: int, table: Optional[np.ndarray]) -> Optional[Tuple[int, int]]:
    if t < 0:
        return None
    p = off + t
    b = p // block_size if table is None else int(table[p // block_size])
    return (b, p % block_size) if 0 <= b < num_blocks else None


def quantise(x: np.ndarray) -> Tuple[np.ndarray, float]:
    """Codes and scale of one row, in the float32 operations that define them."""
    x = x.astype(np.float32)
    if not np.all(np.isfinite(x)):
        return np.zeros(x.shape, np.int8), math.nan
    top = np.float32(np.max(np.abs(x)))
    if top < 2.0 ** -100:
        return np.zeros(x.shape, np.int8), 0.0
    inv = np.float32(127.0) / top
    return np.rint(x * inv).astype(np.int8), float(top / np.float32(127.0))


def attend_rows(q: np.ndarray, k: np.ndarray, v: np.ndarray, there: np.ndarray, scale: float, causal: bool, window: int):
    """q [Q, d] are the last Q of k's / v's [T, d] tokens.  Returns out [Q, d], lse [Q], and for error bounds the
    weighted mean of |v| [Q, d], the largest sum |q k| |scale| [Q] and the largest |score| [Q] over what is seen."""
    Q, d = q.shape
    T = k.shape[0]
    out, mean = np.zeros((Q, d)), np.zeros((Q, d))
    lse, mass, peak = np.full(Q, -np.inf), np.zeros(Q), np.zeros(Q)
    for j in range(Q):
        pos = T - Q + j
        t = np.arange(T)
        see = there & (t <= pos if causal else np.full(T, pos >= 0))
        if window:
            see &= t > pos - window
        if not see.any():
            continue
        with np.errstate(all="ignore"):
            s = scale * (k[see] @ q[j])
            m = np.max(s)
            if m == -np.inf:
                continue
            p = np.exp(s - m)
            out[j] = (p @ v[see]) / p.sum()
            mean[j] = (p @ np.abs(v[see])) / p.sum()
            lse[j] = m + math.log(p.sum()) if np.isfinite(p.sum()) else math.nan
            mass[j] = abs(scale) * np.max(np.abs(k[see]) @ np.abs(q[j]))
            peak[j] = np.max(np.abs(s))
    return out, lse, mean, mass, peak


def attend(q: np.ndarray, kpool: np.ndarray, vpool: np.ndarray, new: Sequence[int], ctx: Sequence[int],
           offs: Sequence[int], tables: Optional[np.ndarray], scale: float, causal: bool = True, window: int = 0):
    """q [N, Hq, d]; pools [nb, bs, H, d] (values, float64).  The arrays of attend_rows, [N, Hq, ...], plus the number
    of tokens in the context [N, Hq]."""
    N, Hq, d = q.shape
    nb, bs, H, _ = kpool.shape
    res = [np.zeros((N, Hq, d)), np.zeros((N, Hq)), np.zeros((N, Hq, d)), np.zeros((N, Hq)), np.zeros((N, Hq))]
    count = np.zeros((N, Hq))
    a = 0
    for i, (n, c) in enumerate(zip(new, ctx)):
        pl: List[Optional[Tuple[int, int]]] = [place(t, offs[i], bs, nb, None if tables is None else tables[i])
                                               for t in range(c)]
        there = np.array([x is not None for x in pl], dtype=bool)
        b = np.array([0 if x is None else x[0] for x in pl], dtype=np.int64)
        s = np.array([0 if x is None else x[1] for x in pl], dtype=np.int64)
        for h in range(Hq):
            k, v = kpool[b, s, h // (Hq // H)], vpool[b, s, h // (Hq // H)]
            if c < n:  # tokens before the context: no place, and nothing to see
                pad = n - c
                k, v = (np.concatenate([np.zeros((pad, d)), x]) for x in (k, v))
                seen = np.concatenate([np.zeros(pad, bool), there])
                part = attend_rows(q[a:a + n, h], k, v, seen, scale, causal, window)
                for x in part[:1] + part[2:]:
                    x[:pad] = 0.0
                part[1][:pad] = -np.inf
            else:
                part = attend_rows(q[a:a + n, h], k, v, there, scale, causal, window)
            for x, y in zip(res, part):
                x[a:a + n, h] = y
            count[a:a + n, h] = c
        a += n
    return (*res, count)
