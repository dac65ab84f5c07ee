"""Trees of drafted tokens for the tests."""
from __future__ import annotations

import numpy as np
import torch

DEV = "cuda"
TREES = ["chain", "levels", "depth", "star", "forest"]


def tree(kind: str, q: int, rng: np.random.Generator) -> np.ndarray:
    """Parents of q tokens."""
    if kind == "chain":
        return np.arange(-1, q - 1)
    if kind == "star":
        return np.array([-1] + [0] * (q - 1))[:q]
    par = np.full(q, -1)
    for j in range(1, q):
        if kind == "levels":
            par[j] = (j - 1) // 3
        elif kind == "depth":
            par[j] = j - 1 if rng.random() < 0.7 else rng.integers(0, j)
        else:  # several trees beside one another
            par[j] = rng.integers(-1, j)
    return par


def i32(x) -> torch.Tensor:
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def i64(x: np.ndarray) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(x).view(np.int64)).to(DEV)
