"""Contexts moved from one cache into another (serving.park), between every two types that go together."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as SO
from paper_2609_34060_amd import kvc, serving

pytestmark = pytest.mark.gpu
DEV = "cuda"
L, H, D, BS = 3, 2, 64, 16


def make(dtype, blocks):
    if dtype == torch.int8:
        return serving.int8_cache(L, blocks, BS, H, D, DEV)
    p = torch.zeros(L, 2, blocks, BS, H, D, dtype=dtype, device=DEV)
    return kvc.Cache(list(p[:, 0]), list(p[:, 1]))


def rows(cache, tables, offsets, lengths):
    """What the cache holds of each sequence, [layers, 2, tokens, H, D], in the pools' type, with the scales in 8 bits."""
    out = []
    for i, n in enumerate(lengths):
        p = torch.arange(n) + offsets[i]
        b, s = tables[i].cpu().long()[p // BS].to(DEV), (p % BS).to(DEV)
        x = torch.stack([torch.stack([cache.k_pools[l][b, s], cache.v_pools[l][b, s]]) for l in range(L)])
        if cache.scales is None:
            out.append(x)
        else:
            out.append((x, torch.stack([torch.stack([cache.k_scales[l][b, s], cache.v_scales[l][b, s]])
                                        for l in range(L)])))
    return out


def tables_of(lengths, offsets, g):
    blocks = [-(-(n + o) // BS) for n, o in zip(lengths, offsets)]
    order = torch.randperm(sum(blocks), generator=g).to(torch.int32).tolist()
    tab = torch.full((len(lengths), max(blocks)), -1, dtype=torch.int32)
    for i, b in enumerate(blocks):
        tab[i, :b] = torch.tensor([order.pop() for _ in range(b)], dtype=torch.int32)
    return tab.to(DEV), sum(blocks)


def filled(dtype, lengths, offsets, g):
    tab, blocks = tables_of(lengths, offsets, g)
    cache = make(dtype, blocks)
    x = torch.randn(2, L, sum(lengths), H, D, generator=g).to(DEV)
    x = x.to(torch.bfloat16 if dtype == torch.bfloat16 else torch.float32)
    kvc.kvc_append(cache, kvc.Step(lengths, lengths, tab, offsets), x[0], x[1])
    return cache, tab


def quantised(x):
    """Codes and scales of rows, row by row, by the definition."""
    flat = x.float().cpu().reshape(-1, D)
    both = [SO.quantise(r.numpy()) for r in flat]
    return (torch.from_numpy(np.stack([c for c, _ in both])).view(x.shape).to(DEV),
            torch.tensor([s for _, s in both], dtype=torch.float32).view(x.shape[:-1]).to(DEV))


LENGTHS, FROM, TO = [37, 1, 100], [3, 0, 17], [0, 15, 5]


@pytest.mark.parametrize("source,target", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                           (torch.float32, torch.int8), (torch.bfloat16, torch.int8),
                                           (torch.int8, torch.float32), (torch.int8, torch.bfloat16),
                                           (torch.int8, torch.int8)])
def test_types(source, target):
    g = torch.Generator().manual_seed(5)
    a, at = filled(source, LENGTHS, FROM, g)
    to, blocks = tables_of(LENGTHS, TO, g)
    b = make(target, blocks)
    serving.park(a, at, FROM, b, to, TO, LENGTHS, layers_at_once=2)
    for was, now in zip(rows(a, at, FROM, LENGTHS), rows(b, to, TO, LENGTHS)):
        if source == torch.int8:
            was = was[0].float() * was[1][..., None]
            was = was.to(torch.float32 if target == torch.float32 else torch.bfloat16)
        if target == torch.int8:
            code, scale = quantised(was)
            assert torch.equal(now[0], code) and torch.equal(now[1], scale)
        else:
            assert torch.equal(now, was)


def test_types_that_do_not_go_together():
    g = torch.Generator().manual_seed(5)
    a, at = filled(torch.float32, LENGTHS, FROM, g)
    to, blocks = tables_of(LENGTHS, TO, g)
    with pytest.raises(kvc.KvcError):
        serving.park(a, at, FROM, make(torch.bfloat16, blocks), to, TO, LENGTHS)
