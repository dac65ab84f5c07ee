"""A turn over a corrected context: fit and apply make the later agent's context, the served step runs its prompt and its
tokens over it, and the context goes into an 8-bit cache and back; every attention against the float64 oracle on the
cache that it was given.

Bounds: one attention as in the served step's tests, here with bfloat16 inputs of standard scale: weights and results
rounded to bfloat16 (2^-9 of the mean |v|, 2^-9 of the result), scores off by (d + 4) 2^-24 sum |q k| (below 2^-13 of a
weight), taken twice and once more for the residual's rounding.  A parked row comes back as its codes
times its scale, rounded once, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as SO
from paper_2609_34060_amd import kvc, pipelines, serving, synth

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Model:
    """Random projections of a few layers, in bfloat16 with float32 products; it keeps what each layer attended with."""

    def __init__(self, L, H, group, d, width=96, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.H, self.heads, self.d = H, H * group, d
        n = (self.heads + 2 * H) * d
        self.w = [(torch.randn(width, n, generator=g) / width ** 0.5).to(DEV) for _ in range(L)]
        self.back = [(torch.randn(self.heads * d, width, generator=g) / (self.heads * d) ** 0.5).to(DEV)
                     for _ in range(L)]
        self.seen = []

    def project(self, layer, x):
        p = (x @ self.w[layer]).to(torch.bfloat16).view(x.shape[0], self.heads + 2 * self.H, self.d)
        q, k, v = p[:, :self.heads], p[:, self.heads:self.heads + self.H], p[:, self.heads + self.H:]
        self.seen.append([layer, q])
        return q, k, v

    def finish(self, layer, x, attended):
        self.seen[-1].append(attended)
        return x + attended.reshape(x.shape[0], -1).float() @ self.back[layer]


def check_turn(model, cache, step, tables, offs, new, ctx):
    k, v = ([values(cache, kv, l) for l in range(cache.num_layers)] for kv in range(2))
    for layer, q, got in model.seen:
        ref, _, mean, mass, peak, n = SO.attend(q.double().cpu().numpy(), k[layer], v[layer], new, ctx, offs, tables,
                                                model.d ** -0.5, True, 0)
        bound = 3 * (2.0 ** -9 * mean + 2.0 ** -9 * np.abs(ref) + 2.0 ** -13 * mean) + 1e-30
        assert np.all(np.abs(got.double().cpu().numpy() - ref) <= bound)
    model.seen.clear()


def values(cache, kv, layer):
    x = (cache.v_pools if kv else cache.k_pools)[layer].double().cpu()
    if cache.scales is not None:
        x = x * (cache.v_scales if kv else cache.k_scales)[layer].double().cpu().unsqueeze(-1)
    return x.numpy()


def test_a_turn_over_a_corrected_context_and_its_parking():
    w = synth.WORKLOADS["tiny"].with_(num_agents=2, num_layers=2, dtype="bf16")
    pc = synth.build_paged(w, device=DEV, num_output_agents=1)
    cache = kvc.Cache(pc.k_pools, pc.v_pools)
    H, d, bs, T = w.num_kv_heads, w.head_dim, w.block_size, w.seq_tokens[0]

    def seq(name):
        s = pc.seqs[name]
        return s.offset, None if pc.tables is None else pc.tables[[s.table_row]]

    # the later agent's context: the earlier one's cache and the fitted transition
    src, dst, out = seq((0, 0)), seq((0, 1)), seq((0, 100))
    pipelines.apply(cache, src, out, T, pipelines.fit(cache, src, dst, T, w.rank))

    # its own pools: the context copied over, with room for what it reads and produces
    blocks = -(-(T + 64) // bs)
    pools = torch.zeros(2, 2, blocks + 3, bs, H, d, dtype=torch.bfloat16, device=DEV)
    own = kvc.Cache(list(pools[0]), list(pools[1]))
    order = torch.randperm(blocks + 3, generator=torch.Generator().manual_seed(3))[:blocks]
    tables = order.to(torch.int32).unsqueeze(0).to(DEV)
    serving.park(cache, out[1], [out[0]], own, tables, None, [T], layers_at_once=1)
    for layer in range(2):
        for kv, pool in enumerate((pc.k_pools[layer], pc.v_pools[layer])):
            s = pc.seqs[(0, 100)]
            at = torch.arange(T) + s.offset
            blk = at // bs if pc.tables is None else pc.tables[s.table_row].cpu().long()[at // bs]
            now = torch.arange(T)
            assert torch.equal(pools[kv, layer][order[now // bs].to(DEV), (now % bs).to(DEV)],
                               pool[blk.to(DEV), (at % bs).to(DEV)])

    # a prompt chunk, then single tokens, with one workspace
    model = Model(2, H, 4, d)
    g = torch.Generator().manual_seed(7)
    tab, at = tables.cpu().numpy(), T
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    for new in (37, 1, 1):
        at += new
        step = kvc.Step([new], [at], tables)
        x = torch.randn(new, 96, generator=g).to(DEV)
        y = serving.forward(own, step, x, model.project, model.finish, workspace=ws)
        assert y.shape == x.shape and bool(torch.isfinite(y).all())
        check_turn(model, own, step, tab, [0], [new], [at])

    # parked in 8 bits, attended with there, and back
    held = serving.int8_cache(2, blocks + 2, bs, H, d, DEV)
    htab = torch.randperm(blocks + 2, generator=g)[:blocks].to(torch.int32).unsqueeze(0).to(DEV)
    serving.park(own, tables, None, held, htab, None, [at])
    step = kvc.Step([1], [at + 1], htab)
    serving.forward(held, step, torch.randn(1, 96, generator=g).to(DEV), model.project, model.finish)
    check_turn(model, held, step, htab.cpu().numpy(), [0], [1], [at + 1])
    again = torch.zeros_like(pools)
    back = kvc.Cache(list(again[0]), list(again[1]))
    serving.park(held, htab, None, back, tables, None, [at])
    now = torch.arange(at)
    place = (slice(None), slice(None), order[now // bs].to(DEV), (now % bs).to(DEV))
    was, got = pools[place].cpu(), again[place].cpu()
    want = torch.empty_like(was)
    for row, to in zip(was.reshape(-1, d), want.view(-1, d)):
        code, scale = SO.quantise(row.float().numpy())
        to.copy_(torch.from_numpy(code).float() * scale)  # (float32 products, rounded once)
    assert torch.equal(got, want)
    assert not torch.equal(got, was)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_more_sequences_than_a_grid_is_deep(kind):
    """70001 single tokens, each over its own context of one (its value) or, every third, two equal keys (the mean)."""
    n, d = 70001, 64
    g = torch.Generator().manual_seed(2)
    pools = torch.randn(2, 2 * n, 1, 1, d, generator=g).to(kind).to(DEV)
    pools[0, 1::2] = pools[0, 0::2]
    cache = kvc.Cache([pools[0]], [pools[1]])
    tables = torch.randperm(n, generator=g).to(torch.int32).to(DEV)[:, None] * 2 + torch.arange(2, device=DEV,
                                                                                              dtype=torch.int32)
    ctx = [2 if i % 3 == 0 else 1 for i in range(n)]
    q = torch.randn(n, 1, d, generator=g).to(kind).to(DEV)
    out = kvc.kvc_attend(cache, kvc.Step([1] * n, ctx, tables), q)
    v = pools[1, :, 0, 0].float()[tables.long()]
    two = torch.arange(n, device=DEV) % 3 == 0
    want = torch.where(two[:, None], (v[:, 0] + v[:, 1]) / 2, v[:, 0]).to(kind)
    assert torch.equal(out[:, 0], want)
