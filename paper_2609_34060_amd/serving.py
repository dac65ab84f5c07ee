"""An agent's turn over a corrected context: tokens written into its cache and attended with, layer by layer, and its
context parked in an 8-bit cache while other agents take theirs.

A later agent's context is materialised by kvc_apply from the cache of an earlier one; from there on the agent reads its
own prompt and produces tokens over that context.  `forward` is one step of that (a chunk of a prompt, one token for
each sequence, or both in one batch); the projections around the attention are the caller's.  `park` moves contexts
from one cache into another of any dtype: into int8 to hold 1.94 times the contexts (head_dim 128) in the same memory,
and back into a bfloat16 or float32 cache where a fit or a correction is to read them (those take no 8-bit rows).
"""
from __future__ import annotations

from typing import Callable, Optional, Sequence, Tuple

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


def park(source: kvc.Cache, source_tables: Optional[torch.Tensor], source_offsets: Optional[Sequence[int]],
         target: kvc.Cache, target_tables: Optional[torch.Tensor], target_offsets: Optional[Sequence[int]],
         num_tokens: Sequence[int], dtype: Optional[torch.dtype] = None, layers_at_once: int = 8) -> None:
    """Copies the first num_tokens[i] tokens of every sequence i into another cache of the same heads and layers, by way
    of rows of `dtype` for layers_at_once layers at a time.  The dtype is that of the cache which is not int8 (bfloat16
    where both are); a bfloat16 and a float32 cache do not go together."""
    dev = source.k_pools[0].device
    if dtype is None:
        held = [c.k_pools[0].dtype for c in (source, target) if c.c.dtype != kvc.KVC_I8]
        dtype = held[0] if held else torch.bfloat16
    read = kvc.Step(num_tokens, num_tokens, source_tables, source_offsets, device=dev)
    write = kvc.Step(num_tokens, num_tokens, target_tables, target_offsets, device=dev)
    c = source.c
    # (rows whose table entry names no block are left as they are by the read: zeros)
    rows = torch.zeros(2, min(layers_at_once, c.num_layers), read.num_rows, c.num_kv_heads, c.head_dim, dtype=dtype,
                       device=dev)
    for at in range(0, c.num_layers, layers_at_once):
        end = min(at + layers_at_once, c.num_layers)
        k, v = rows[0, :end - at], rows[1, :end - at]
        kvc.kvc_gather(source, read, k, v, at, end)
        kvc.kvc_append(target, write, k, v, at, end)
