"""A step of drafted tokens in float64, written from the definitions (test infrastructure only).

A sequence's new tokens are numbered from 0; parents[j] is the one that token j continues, or -1 (it continues the context
before them)."""
from __future__ import annotations

import math
from typing import List, Optional, Sequence, Tuple

import numpy as np

from oracle.serve_oracle import place


def line_of(parents: Sequence[int], j: int) -> Optional[List[int]]:
    """Token j and its ancestors, or None where its line does not end at -1 through earlier tokens."""
    line = [j]
    while parents[line[-1]] != -1:
        p = parents[line[-1]]
        if p < -1 or p >= line[-1]:
            return None
        line.append(p)
    return line


def tree(parents: Sequence[int], base: int, words: int) -> Tuple[np.ndarray, np.ndarray]:
    """Masks [q, words] (uint64) and positions [q] of a sequence whose context before the new tokens has `base` tokens."""
    masks, positions = np.zeros((len(parents), words), np.uint64), np.full(len(parents), -1, np.int64)
    for j in range(len(parents)):
        line = line_of(parents, j)
        if line is None:
            continue
        for v in line:
            masks[j, v // 64] |= np.uint64(1 << (v % 64))
        positions[j] = base + len(line) - 1
    return masks, positions


def rotate(x: np.ndarray, positions: np.ndarray, inv_freq: np.ndarray, pairs: bool, factor: float, inverse: bool = False):
    """x [N, heads, d] (float64).  Angles in extended precision, so that they hold at any position."""
    r = 2 * len(inv_freq)
    turns = positions.astype(np.longdouble)[:, None] * (inv_freq.astype(np.longdouble) / (2 * np.arccos(np.longdouble(-1))))
    angle = ((turns - np.rint(turns)) * (2 * np.arccos(np.longdouble(-1)))).astype(np.float64) * (-1.0 if inverse else 1.0)
    c, s = factor * np.cos(angle)[:, None], factor * np.sin(angle)[:, None]
    a, b = (slice(0, r, 2), slice(1, r, 2)) if pairs else (slice(0, r // 2), slice(r // 2, r))
    y = x.copy()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def bits(masks: np.ndarray, q: int) -> np.ndarray:
    """[q, q] truth values of a sequence's masks [q, words] (int64 or uint64)."""
    w = masks.view(np.uint64)
    return np.array([[bool((int(w[i, j // 64]) >> (j % 64)) & 1) for j in range(q)] for i in range(q)], dtype=bool).reshape(q, q)


def attend(q: np.ndarray, kpool: np.ndarray, vpool: np.ndarray, new: Sequence[int], ctx: Sequence[int],
           offs: Sequence[int], tables: Optional[np.ndarray], masks: np.ndarray, scale: float, window: int = 0):
    """q [N, Hq, d]; pools [nb, bs, H, d] (values, float64).  out [N, Hq, d], lse [N, Hq], and for error bounds the weighted
    mean of |v| [N, Hq, d], and [N, Hq] each: the largest sum |q k| |scale|, the largest |score|, how many are seen."""
    N, Hq, d = q.shape
    nb, bs, H, _ = kpool.shape
    out, mean = np.zeros((N, Hq, d)), np.zeros((N, Hq, d))
    lse, mass, peak, seen = np.full((N, Hq), -np.inf), np.zeros((N, Hq)), np.zeros((N, Hq)), np.zeros((N, Hq))
    at = 0
    for i, (n, c) in enumerate(zip(new, ctx)):
        base, sees = c - n, bits(masks[at:at + n], n)
        where = [place(t, offs[i], bs, nb, None if tables is None else tables[i]) for t in range(c)]
        for j in range(n):
            if base + j < 0:
                continue
            p = base - 1 + int(sees[j].sum())
            t = [x for x in range(c) if where[x] is not None and
                 (sees[j, x - base] if x >= base else not window or x > p - window)]
            if not t:
                continue
            b, s = np.array([where[x][0] for x in t]), np.array([where[x][1] for x in t])
            for h in range(Hq):
                k, v = kpool[b, s, h // (Hq // H)], vpool[b, s, h // (Hq // H)]
                with np.errstate(all="ignore"):
                    z = scale * (k @ q[at + j, h])
                    m = z.max()
                    if m == -np.inf:
                        continue
                    w = np.exp(z - m)
                    out[at + j, h], mean[at + j, h] = (w @ v) / w.sum(), (w @ np.abs(v)) / w.sum()
                    lse[at + j, h] = m + math.log(w.sum()) if np.isfinite(w.sum()) else math.nan
                    mass[at + j, h] = abs(scale) * np.max(np.abs(k) @ np.abs(q[at + j, h]))
                    peak[at + j, h], seen[at + j, h] = np.max(np.abs(z)), len(t)
        at += n
    return out, lse, mean, mass, peak, seen


def weights(row: np.ndarray) -> np.ndarray:
    """A row of probabilities as it counts."""
    x = row.astype(np.float64)
    return np.where((x > 0) & np.isfinite(x), x, 0.0)


def number(u: float) -> float:
    """A random number as it counts."""
    return 0.0 if math.isnan(u) else min(max(u, 0.0), 1.0 - 2.0 ** -24)


def verify(parents, tokens, target, draft, uniforms, last: float, children: int = 0):
    """One sequence: rows target (and draft) [q, V].  The accepted tokens and the next one, -1 where there is none."""
    path, tried = [0], 0
    P = weights(target[0])
    Q = None if draft is None else weights(draft[0])
    left, whole = P.copy(), 1.0  # what is left to draw from, as the residuals' definition has it, and its sum
    for j in range(1, len(parents)):
        if parents[j] != path[-1] or (children and tried == children):
            continue
        x, u = int(tokens[j]), number(float(uniforms[j]))
        there = 0 <= x < len(P)
        r = left[x] if there else 0.0
        if u * whole * (1.0 if Q is None else Q[x] if there else 0.0) < r:
            path.append(j)
            P, tried = weights(target[j]), 0
            Q = None if draft is None else weights(draft[j])
            left, whole = P.copy(), 1.0
            continue
        tried += 1
        if Q is None:
            whole = max(0.0, whole - r)
            if there:
                left[x] = 0.0
        else:
            left = np.maximum(0.0, left - whole * Q)
            whole = math.fsum(left)
    if not left.any():
        left = P
    if not left.any():
        return path, -1
    share, run = number(float(last)) * math.fsum(left), 0.0
    for x in np.nonzero(left)[0]:
        run += left[x]
        if run > share:
            return path, int(x)
    return path, int(np.nonzero(left)[0][-1])


def keep(path: Sequence[int], count: int, q: int) -> List[Tuple[int, int]]:
    """(from, to) of the new tokens that move, in order."""
    moves, before = [], -1
    for d in range(min(count, q)):
        if path[d] <= before or path[d] >= q:
            break
        before = path[d]
        if path[d] != d:
            moves.append((path[d], d))
    return moves
