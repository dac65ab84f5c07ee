"""An agent's turn over a corrected context: tokens written into its cache and attended with, layer by layer, and its
context parked in an 8-bit cache while other agents take theirs.

A later agent's context is materialised by kvc_apply from the cache of an earlier one; from there on the agent reads its
own prompt and produces tokens over that context.  `forward` is one step of that (a chunk of a prompt, one token for
each sequence, or both in one batch); the projections around the attention are the caller's.  `park` moves contexts
from one cache into another of any dtype: into int8 to hold 1.94 times the contexts (head_dim 128) in the same memory,
and back into a bfloat16 or float32 cache where a fit or a correction is to read them (those take no 8-bit rows).
"""
from __future__ import annotations

import itertools
from typing import Callable, List, Optional, Sequence, Tuple

import torch

from . import kvc

Project = Callable[[int, torch.Tensor], Tuple[torch.Tensor, torch.Tensor, torch.Tensor]]
Finish = Callable[[int, torch.Tensor, torch.Tensor], torch.Tensor]


def int8_cache(num_layers: int, num_blocks: int, block_size: int, num_kv_heads: int, head_dim: int, device) -> kvc.Cache:
    """An 8-bit cache: pools [layers, K/V, blocks, block_size, heads, head_dim] and scales with a head's tokens next to
    one another, as attention reads them."""
    pools = torch.zeros(num_layers, 2, num_blocks, block_size, num_kv_heads, head_dim, dtype=torch.int8, device=device)
    scales = torch.zeros(num_layers, 2, num_blocks, num_kv_heads, block_size, device=device).transpose(-1, -2)
    return kvc.Cache(list(pools[:, 0]), list(pools[:, 1]), k_scales=list(scales[:, 0]), v_scales=list(scales[:, 1]))


def forward(cache: kvc.Cache, step: kvc.Step, x: torch.Tensor, project: Project, finish: Finish, window: int = 0,
            scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One step through every layer.  project(layer, x) gives q [N, heads, head_dim], k and v [N, num_kv_heads, head_dim]
    (keys rotated to their positions where the model rotates them; views of one packed projection are fine);
    finish(layer, x, attended) gives the layer's output.  A given workspace serves all layers and later steps under the
    same bounds (kvc_attend_workspace_bytes), so that nothing is allocated here."""
    for layer in range(cache.num_layers):
        q, k, v = project(layer, x)
        kvc.kvc_append(cache, step, k, v, layer, layer + 1)
        x = finish(layer, x, kvc.kvc_attend(cache, step, q, layer=layer, scale=scale, window=window,
                                            workspace=workspace))
    return x


def _pieces(num_tokens: Sequence[int], at_once: int) -> List[List[Tuple[int, int, int]]]:
    """The tokens of all sequences in order, (sequence, first, end), cut into pieces of at most at_once tokens."""
    pieces, room = [[]], at_once
    for i, n in enumerate(num_tokens):
        first = 0
        while first < n:
            if room == 0:
                pieces.append([])
                room = at_once
            end = min(n, first + room)
            pieces[-1].append((i, first, end))
            room -= end - first
            first = end
    return [p for p in pieces if p]


def park(source: kvc.Cache, source_tables: Optional[torch.Tensor], source_offsets: Optional[Sequence[int]],
         target: kvc.Cache, target_tables: Optional[torch.Tensor], target_offsets: Optional[Sequence[int]],
         num_tokens: Sequence[int], dtype: Optional[torch.dtype] = None, layers_at_once: int = 8,
         tokens_at_once: int = 65536) -> None:
    """Copies the first num_tokens[i] tokens of every sequence i into another cache of the same heads and layers, by way
    of rows of `dtype` for layers_at_once layers and tokens_at_once tokens at a time, which is all the memory that is taken
    (2 GiB for eight bfloat16 heads of 128; 64 contexts of 8192 tokens of eight layers into int8: 13.7 ms, 14.4 with a
    quarter of the tokens).  The dtype is that of the cache which is not int8 (bfloat16 where both are);
    a bfloat16 and a float32 cache do not go together."""
    dev = source.k_pools[0].device
    if dtype is None:
        held = [c.k_pools[0].dtype for c in (source, target) if c.c.dtype != kvc.KVC_I8]
        dtype = held[0] if held else torch.bfloat16
    if tokens_at_once < 1 or layers_at_once < 1:
        raise ValueError("at least one token and one layer at a time")
    for t, o in ((source_tables, source_offsets), (target_tables, target_offsets)):
        if (t is not None and t.shape[0] != len(num_tokens)) or (o is not None and len(o) != len(num_tokens)):
            raise ValueError("one row of the tables and one offset for each sequence")

    caches = [(None if t is None else t.to(torch.int32).contiguous(), o) for t, o in
              ((source_tables, source_offsets), (target_tables, target_offsets))]
    # the lengths of all pieces go to the device in one copy, before there is work that it would wait for
    plans, host = [], []

    def put(values):
        host.extend(int(x) for x in values)
        return len(host) - len(values), len(host)

    for piece in _pieces(num_tokens, tokens_at_once):
        s0, s1 = piece[0][0], piece[-1][0] + 1
        parts = {i: (end - first, end) for i, first, end in piece}
        new, upto = zip(*[parts.get(i, (0, 0)) for i in range(s0, s1)])
        plans.append((s0, s1, new, upto, put([0, *itertools.accumulate(new)]), put(upto),
                      [None if o is None else put(o[s0:s1]) for _, o in caches]))
    lengths = torch.tensor(host, dtype=torch.int32, device=dev)
    steps = []
    for s0, s1, new, upto, starts, contexts, offsets in plans:
        steps.append([kvc.Step.on_device(lengths[slice(*starts)], lengths[slice(*contexts)], sum(new), max(new), max(upto),
                                         None if t is None else t[s0:s1], None if at is None else lengths[slice(*at)])
                      for (t, _), at in zip(caches, offsets)])
    c = source.c
    buffer = torch.empty(2, min(layers_at_once, c.num_layers), max((r.num_rows for r, _ in steps), default=0),
                         c.num_kv_heads, c.head_dim, dtype=dtype, device=dev)
    for read, write in steps:
        rows = buffer[:, :, :read.num_rows].zero_()  # (those whose table entry names no block are left by the read)
        for at in range(0, c.num_layers, layers_at_once):
            end = min(at + layers_at_once, c.num_layers)
            k, v = rows[0, :end - at], rows[1, :end - at]
            kvc.kvc_gather(source, read, k, v, at, end)
            kvc.kvc_append(target, write, k, v, at, end)
