"""Steps of drafted tokens as they are used, one after the other, against the same tokens decoded one at a time."""
import numpy as np
import pytest
import torch

from paper_2609_34060_amd import kvc, serving
from tests.draft_helpers import DEV, i32, tree

pytestmark = pytest.mark.gpu
L, H, HQ, D, V, BS = 2, 2, 8, 64, 37, 16


class Model:
    """A small decoder in the rows' type: embedding, two attention layers with residuals, rotary positions, logits."""

    def __init__(self, dtype, seed=0):
        g = torch.Generator().manual_seed(seed)
        w = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale / s[0] ** 0.5).to(DEV)
        self.dtype, self.width = dtype, HQ * D
        self.embed = torch.randn(V, self.width, generator=g).to(DEV)
        self.qkv = [w(self.width, (HQ + 2 * H) * D) for _ in range(L)]
        self.o = [w(self.width, self.width) for _ in range(L)]
        self.head = w(self.width, V, scale=4.0)
        self.rotary = kvc.Rotary(kvc.rope_frequencies(32), D)

    def project(self, layer, x):
        y = (x @ self.qkv[layer]).view(-1, HQ + 2 * H, D).to(self.dtype)
        return y[:, :HQ], y[:, HQ:HQ + H], y[:, HQ + H:]

    def finish(self, layer, x, attended):
        return x + attended.float().reshape(x.shape) @ self.o[layer]

    def probabilities(self, cache, step, tokens, positions, masks=None, workspace=None):
        x = serving.forward(cache, step, self.embed[tokens.long()], self.project, self.finish, masks=masks,
                            rotary=self.rotary, positions=positions, workspace=workspace)
        return torch.softmax(x @ self.head, -1)


def cache_of(kind, blocks):
    if kind == "i8":
        return serving.int8_cache(L, blocks, BS, H, D, DEV)
    dt = torch.bfloat16 if kind == "bf16" else torch.float32
    pools = torch.zeros(L, 2, blocks, BS, H, D, dtype=dt, device=DEV)
    return kvc.Cache(list(pools[:, 0]), list(pools[:, 1]))


def decode(model, kind, prompts, texts):
    """The probabilities after every token of the texts, one token at a time behind the prompts."""
    n = len(prompts)
    cache, tables = cache_of(kind, 8 * n), torch.arange(8 * n, dtype=torch.int32, device=DEV).view(n, 8)
    sizes = [len(p) for p in prompts]
    pos = np.concatenate([np.arange(s) for s in sizes])
    model.probabilities(cache, kvc.Step(sizes, sizes, tables), i32(np.concatenate(prompts)), i32(pos))
    res = [[] for _ in prompts]
    for t in range(max(len(x) for x in texts)):
        live = [i for i in range(n) if t < len(texts[i])]
        step = kvc.Step([1] * len(live), [sizes[i] + t + 1 for i in live], tables[live])
        p = model.probabilities(cache, step, i32([texts[i][t] for i in live]), i32([sizes[i] + t for i in live]))
        for r, i in enumerate(live):
            res[i].append(p[r])
    return [torch.stack(x) for x in res]


@pytest.mark.parametrize("kind,drawn,children", [("f32", True, 0), ("f32", True, 1), ("f32", False, 0), ("bf16", True, 0),
                                                 ("bf16", False, 0), ("i8", True, 0), ("i8", False, 0)])
def test_speculation_is_decoding(kind, drawn, children):
    """Twelve steps of trees of up to 12 tokens: the target's probabilities along the accepted tokens are those of the same
    text decoded a token at a time, and so are the keys and values that were kept."""
    model = Model(torch.float32 if kind == "f32" else torch.bfloat16)
    n, rng, g = 3, np.random.default_rng(4), torch.Generator().manual_seed(6)
    prompts = [rng.integers(0, V, size=s) for s in (5, 16, 23)]
    cache = cache_of(kind, 8 * n)
    tables = torch.randperm(8 * n, generator=g).to(torch.int32).view(n, 8).to(DEV)
    ctx = [len(p) for p in prompts]
    model.probabilities(cache, kvc.Step(ctx, ctx, tables), i32(np.concatenate(prompts)),
                        i32(np.concatenate([np.arange(s) for s in ctx])))
    texts, probs = [[int(p[0])] for p in prompts], [[] for _ in prompts]  # (token 0 of the first step: any)
    for s in range(12):
        sizes = [int(rng.integers(1, 13)) for _ in range(n)]
        parents = [tree(["levels", "depth", "chain", "star"][(s + i) % 4], q, rng) for i, q in enumerate(sizes)]
        par = i32(np.concatenate(parents))
        step = kvc.Step(sizes, [c + q for c, q in zip(ctx, sizes)], tables)
        masks, positions = kvc.kvc_tree(step, par)
        starts = np.cumsum([0] + sizes)
        # half of the vocabulary, the same at every token: far enough from the target to reject, near enough to accept
        draft = torch.zeros(int(starts[-1]), V)
        draft[:, : V // 2] = 1.0 / (V // 2)
        tokens = torch.randint(0, V // 2, (int(starts[-1]),), generator=g).to(torch.int32)
        for i in range(n):
            tokens[starts[i]] = texts[i][-1]
        target = model.probabilities(cache, step, tokens.to(DEV), positions, masks)
        path, counts, chosen = serving.settle(
            cache, step, par, tokens.to(DEV), target, torch.rand(int(starts[-1]), generator=g).to(DEV),
            torch.rand(n, generator=g).to(DEV), draft.to(DEV) if drawn else None, children)
        for i in range(n):
            took = path[starts[i]: starts[i] + int(counts[i])].tolist()
            assert took[0] == 0 and all(parents[i][b] == a for a, b in zip(took, took[1:]))
            texts[i] += [int(tokens[starts[i] + j]) for j in took[1:]] + [int(chosen[i])]
            probs[i] += [target[starts[i] + j] for j in took]
            ctx[i] += len(took)
    assert max(len(t) for t in texts) > 13  # (1 and one a step: some drafts were accepted)
    want = decode(model, kind, prompts, [t[:-1] for t in texts])
    # The plans of the two ways cut and round sums differently: results of one layer to half a step of the rows' type (and
    # a weight's, 2^-8), two layers, logits of up to 4 times the width's root: within 64 steps of it in all.
    eps = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "i8": 2.0 ** -8}[kind]
    for a, b in zip(probs, want):
        assert float((torch.stack(a) - b).abs().max()) <= 64 * eps
    for i in range(n):
        assert ctx[i] == len(prompts[i]) + len(texts[i]) - 1


def test_captured_step():
    """A whole step of speculation in one graph: tree, rotation, append, attention, verification and the rows' moves, replayed
    over changing trees, tokens and lengths and compared with the same calls made one by one."""
    model = Model(torch.bfloat16)
    n, q, g, rng = 2, 8, torch.Generator().manual_seed(3), np.random.default_rng(1)
    caches = [cache_of("bf16", 16) for _ in range(2)]
    tables = torch.arange(16, dtype=torch.int32, device=DEV).view(n, 8)
    for c in caches:
        model.probabilities(c, kvc.Step([30, 40], [30, 40], tables), i32(np.arange(70) % V), i32(np.r_[:30, :40]))
    ctx = i32([38, 48])
    step = kvc.Step.on_device(i32([0, 8, 16]), ctx, 16, 8, 128, tables)
    par, tokens = i32(np.concatenate([tree("levels", 8, rng)] * 2)), i32(np.arange(16) % V)
    uniforms, last = torch.rand(16, generator=g).to(DEV), torch.rand(2, generator=g).to(DEV)
    ws = torch.empty(max(1, kvc.kvc_attend_workspace_bytes(caches[0], step, HQ)), dtype=torch.uint8, device=DEV)
    vs = torch.empty(kvc.kvc_verify_workspace_bytes(step, V), dtype=torch.uint8, device=DEV)

    def turn(cache):
        masks, positions = kvc.kvc_tree(step, par)
        target = model.probabilities(cache, step, tokens, positions, masks, ws)
        return serving.settle(cache, step, par, tokens, target, uniforms, last, workspace=vs)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        turn(caches[0])
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(caches[1].k_pools + caches[1].v_pools, caches[0].k_pools + caches[0].v_pools):
        a.copy_(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = turn(caches[0])
    for s in range(5):
        par.copy_(i32(np.concatenate([tree(k, 8, rng) for k in (("depth", "star"), ("chain", "levels"))[s % 2]])))
        tokens.copy_(torch.randint(0, V, (16,), generator=g))
        uniforms.copy_(torch.rand(16, generator=g) * 0.05)
        last.copy_(torch.rand(2, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        want = turn(caches[1])
        for o, w in zip(out, want):
            assert torch.equal(o, w)
        for a, b in zip(caches[1].k_pools + caches[1].v_pools, caches[0].k_pools + caches[0].v_pools):
            assert torch.equal(a, b)
        ctx.add_(want[1])


def test_forward_refuses_half_a_rotation():
    with pytest.raises(ValueError, match="together"):
        serving.forward(cache_of("f32", 1), None, torch.zeros(1), None, None, rotary=kvc.Rotary([1.0], D))
