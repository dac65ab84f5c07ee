"""Lengths on the device that contradict the host's bounds, starts that descend above all: what they leave out stays as it
was, and what they do not is as without them, in every way that a step is cut into work (a tile a sequence, tiles that
are searched for, ranges that are joined) and for the moves.

Which sequences are left out is worked out here from the definition: starts[i] above starts[i + 1] or below an earlier
start, a start outside [0, N], more new tokens or a longer context than the bounds say."""
import numpy as np
import pytest
import torch

from paper_2609_34060_amd import kvc

pytestmark = pytest.mark.gpu
DEV = "cuda"
H, BS = 2, 16


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def served(starts, ctx, num_rows, max_new, max_context):
    return [i for i in range(len(ctx))
            if 0 <= starts[i] <= starts[i + 1] <= num_rows and starts[i] == max(starts[:i + 1])
            and starts[i + 1] - starts[i] <= max_new and 0 <= ctx[i] <= max_context]


def pools(n, ctx, kind, d, seed=0):
    """Pools with n sequences' blocks in order (sequence i owns blocks i w .. (i + 1) w - 1), and their tables."""
    g = torch.Generator().manual_seed(seed)
    w = -(-ctx // BS)
    x = torch.randn(2, n * w, BS, H, d, generator=g)
    scales = None
    if kind == "i8":
        x = torch.clamp(torch.round(x * 40), -127, 127)
        scales = (0.01 + 0.05 * torch.rand(2, n * w, BS, H, generator=g)).to(DEV)
    x = x.to({"bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8}[kind]).to(DEV)
    return x, scales, torch.arange(n * w, dtype=torch.int32, device=DEV).view(n, w)


def cache_of(x, scales):
    if scales is None:
        return kvc.Cache([x[0]], [x[1]])
    return kvc.Cache([x[0]], [x[1]], k_scales=[scales[0]], v_scales=[scales[1]])


# starts, new tokens at most, contexts.  The numbers of rows (twice as many query as KV heads) make tiles of 16, 128 and 256
# rows; single sequences with long contexts have their ranges joined.
STEPS = {
    "descends_then_rises": ([0, 12, 15, 3, 20], 20, 40),
    "a_later_one_first": ([40, 60, 0, 30], 60, 70),
    "past_the_rows_between": ([0, 4, 1000, 8, 12], 12, 40),
    "negative": ([0, 6, -5, 6, 9], 9, 40),
    "more_than_the_bound": ([0, 3, 40, 44], 8, 50),
    "first_only": ([9, 0, 5, 9], 9, 40),
    "lowest_and_highest": ([0, 7, 2 ** 31 - 1, -2 ** 31, 7, 12], 12, 40),
    "tall": ([400, 500, 0, 100], 500, 600),
    "tall_between": ([0, 150, 290, 20, 300, 400], 400, 500),
    "single_tokens": ([0, 1, 2, 1, 3, 4, 2, 5], 2, 40),
    "long": ([1, 2, 0, 1], 2, 5000),
    "long_tall": ([0, 90, 70, 160, 20], 160, 3000),
    "good": ([0, 5, 5, 9], 9, 40),
}


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("i8", 128), ("f32", 64)])
@pytest.mark.parametrize("name", list(STEPS))
def test_attend(kind, d, name):
    starts, max_new, ctx = STEPS[name]
    n = len(starts) - 1
    N = max(s for s in starts if s < 2 ** 20 and s != 1000)
    x, scales, tables = pools(n, ctx, kind, d)
    cache = cache_of(x, scales)
    q = torch.randn(N, 2 * H, d, generator=torch.Generator().manual_seed(3)).to(
        torch.float32 if kind == "f32" else torch.bfloat16).to(DEV)
    contexts = [ctx - 3 * i for i in range(n)]
    out, lse = torch.full_like(q, 9.0), torch.full((N, 2 * H), 9.0, device=DEV)
    step = kvc.Step.on_device(i32(starts), i32(contexts), N, min(max_new, N), ctx, tables)
    kvc.kvc_attend(cache, step, q, out, lse=lse)
    good = served(starts, contexts, N, min(max_new, N), ctx)
    left = torch.ones(N, dtype=torch.bool, device=DEV)
    for i in good:
        a, z = starts[i], starts[i + 1]
        left[a:z] = False
        if a == z:
            continue
        alone_lse = torch.empty(z - a, 2 * H, device=DEV)
        alone = kvc.kvc_attend(cache, kvc.Step([z - a], [contexts[i]], tables[i:i + 1]), q[a:z].contiguous(), lse=alone_lse)
        # (two orders of the same sums: scores off by e <= (d + 4) 2^-24 14, sums over up to 5000 tokens by 3e-4, so results
        # and lse by twice 2 e + 3e-4 < 2^-9; weights and results rounded to bfloat16 by 2^-8 of values about 1 each)
        tol = 2.0 ** -9 if kind == "f32" else 2.0 ** -6
        assert torch.all((out[a:z].float() - alone.float()).abs() <= tol * (1 + alone.float().abs())), (name, i)
        assert torch.all((lse[a:z] - alone_lse).abs() <= 2.0 ** -9), (name, i)
    assert torch.all(out[left] == 9.0) and torch.all(lse[left] == 9.0)


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("i8", 64), ("f32", 128)])
@pytest.mark.parametrize("name", list(STEPS))
def test_append_and_gather(kind, d, name):
    starts, max_new, ctx = STEPS[name]
    n = len(starts) - 1
    N = max(s for s in starts if s < 2 ** 20 and s != 1000)
    x, scales, tables = pools(n, ctx, kind, d)
    x0, s0 = x.clone(), None if scales is None else scales.clone()
    contexts = [ctx - 3 * i for i in range(n)]
    step = kvc.Step.on_device(i32(starts), i32(contexts), N, min(max_new, N), ctx, tables)
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    k, v = torch.randn(2, N, H, d, generator=torch.Generator().manual_seed(4)).to(dt).to(DEV)
    good = served(starts, contexts, N, min(max_new, N), ctx)

    # what the step holds is read, and nothing else of the rows is touched
    gk, gv = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
    kvc.kvc_gather(cache_of(x, scales), step, gk, gv)
    want_k, want_v = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
    written = torch.zeros(x.shape[1], BS, dtype=torch.bool, device=DEV)
    for i in good:
        for j in range(starts[i + 1] - starts[i]):
            t = contexts[i] - (starts[i + 1] - starts[i]) + j
            if t < 0:
                continue
            b, s = int(tables[i, t // BS]), t % BS
            written[b, s] = True
            for kv, want in enumerate((want_k, want_v)):
                row = x[kv, b, s].float()
                want[starts[i] + j] = (row if scales is None else row * scales[kv, b, s][:, None]).to(dt)
    assert torch.equal(gk, want_k) and torch.equal(gv, want_v)

    # what it holds is written, and nothing else of the pools is touched
    kvc.kvc_append(cache_of(x, scales), step, k, v)
    assert torch.equal(x[:, ~written], x0[:, ~written])
    if scales is not None:
        assert torch.equal(scales[:, ~written], s0[:, ~written])
    gk.fill_(9.0)
    gv.fill_(9.0)
    kvc.kvc_gather(cache_of(x, scales), step, gk, gv)
    for src, got in ((k, gk), (v, gv)):
        for i in good:
            a, z = max(starts[i], starts[i + 1] - contexts[i]), starts[i + 1]
            if kind == "i8":  # within half a scale, and the rounding of the value to bfloat16 (2^-8 of it)
                top = src[a:z].float().abs().amax(-1, keepdim=True)
                assert torch.all((got[a:z].float() - src[a:z].float()).abs() <= 0.51 * top / 127 + top * 2.0 ** -8)
            else:
                assert torch.equal(got[a:z], src[a:z])


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("i8", 128), ("f32", 64)])
@pytest.mark.parametrize("new,ctx", [([12], [7]), ([90, 3], [70, 40]), ([300], [290]), ([2, 1], [1, 5000]), ([5], [0])])
def test_windows_wider_than_every_context(kind, d, new, ctx):
    """They hide nothing, up to the widest that there is, for tokens without a place (fewer tokens in the cache than new
    ones) beside those with one: the same bits as without a window."""
    x, scales, tables = pools(len(new), max(ctx) + 1, kind, d)
    cache, step = cache_of(x, scales), kvc.Step(new, ctx, tables)
    q = torch.randn(sum(new), 2 * H, d, generator=torch.Generator().manual_seed(3)).to(
        torch.float32 if kind == "f32" else torch.bfloat16).to(DEV)
    lse = torch.empty(sum(new), 2 * H, device=DEV)
    out = kvc.kvc_attend(cache, step, q, lse=lse)
    at = 0
    for n, c in zip(new, ctx):
        nothing = max(0, n - c)
        assert torch.all(lse[at:at + nothing] == -float("inf")) and torch.all(lse[at + nothing:at + n] > -1e3)
        at += n
    for window in (max(ctx) + 1, 2 ** 30, 2 ** 31 - 2, 2 ** 31 - 1):
        lse_w = torch.empty_like(lse)
        assert torch.equal(kvc.kvc_attend(cache, step, q, lse=lse_w, window=window), out)
        assert torch.equal(lse_w, lse)


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("i8", 64), ("f32", 64)])
@pytest.mark.parametrize("new,ctx", [([1], 1100), ([1, 1, 1], 2000), ([33], 1601)])
def test_odd_numbers_of_ranges_and_rows(kind, d, new, ctx):
    """Ranges times rows times heads odd: the parts of the ranges in a workspace of exactly the size that is asked for, with
    nothing written behind it."""
    x, scales, tables = pools(len(new), ctx, kind, d)
    x, scales = x[..., :1, :], None if scales is None else scales[..., :1]
    cache, step = cache_of(x, scales), kvc.Step(new, [ctx] * len(new), tables)
    q = torch.randn(sum(new), 5, d, generator=torch.Generator().manual_seed(3)).to(
        torch.float32 if kind == "f32" else torch.bfloat16).to(DEV)
    need = kvc.kvc_attend_workspace_bytes(cache, step, 5)
    assert need > 0 and need % ((sum(new) * 5) * (4 * d + 8)) == 0
    room = torch.full((need + 4096,), 173, dtype=torch.uint8, device=DEV)
    out = kvc.kvc_attend(cache, step, q, workspace=room[:need])
    assert torch.all(room[need:] == 173)
    k, v = (x[i, :, :, 0].double() if scales is None else x[i, :, :, 0].double() * scales[i, :, :, 0, None].double()
            for i in range(2))
    for i, n in enumerate(new):
        ki, vi = (y[tables[i].long()].reshape(-1, d)[:ctx] for y in (k, v))
        at = sum(new[:i])
        s = torch.matmul(q[at:at + n].double().reshape(-1, d), ki.t().contiguous()) * d ** -0.5
        see = torch.arange(ctx, device=DEV) <= torch.arange(ctx - n, ctx, device=DEV)[:, None]
        p = torch.softmax(s.masked_fill(~see.repeat_interleave(5, 0), -float("inf")), -1)
        want, mean = torch.matmul(p, vi), torch.matmul(p, vi.abs())
        # weights and result rounded to bfloat16 by 2^-8 of their mean magnitude; in float32 scores off by e <= 68 2^-24 14,
        # sums over the tokens by 2000 2^-24
        tol = 2.0 ** -11 if kind == "f32" else 2.0 ** -8
        err = (out[at:at + n].double().reshape(-1, d) - want).abs()
        assert torch.all(err <= tol * (mean + want.abs()) + 2.0 ** -11 * mean)


@pytest.mark.parametrize("n", [64, 65, 200, 1000])
def test_more_sequences_than_a_wave_looks_at_together(n):
    """Starts that rise, with sequences of no token among them, then one that lies above all that follow: those are left
    out, whichever group of 64 they are in."""
    rng = np.random.default_rng(n)
    new = rng.integers(0, 3, n)
    starts = np.concatenate([[0], np.cumsum(new)])
    N, ctx, d = int(starts[-1]), 20, 64
    x, scales, tables = pools(n, ctx, "bf16", d)
    q = torch.randn(N, 2 * H, d, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    k = torch.randn(N, H, d, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(DEV)
    whole = kvc.kvc_attend(cache_of(x, scales), kvc.Step.on_device(i32(starts.tolist()), i32([ctx] * n), N, 2, ctx, tables), q)
    for at in (1, n // 3, n - 1):
        s = starts.tolist()
        s[at] = N
        good = served(s, [ctx] * n, N, 2, ctx)
        step = kvc.Step.on_device(i32(s), i32([ctx] * n), N, 2, ctx, tables)
        keep = torch.zeros(N, dtype=torch.bool, device=DEV)
        same = torch.zeros(N, dtype=torch.bool, device=DEV)
        written = torch.zeros(x.shape[1], BS, dtype=torch.bool, device=DEV)
        for i in good:
            keep[s[i]:s[i + 1]] = True
            same[s[i]:s[i + 1]] = i != at - 1  # (that one's end is another now: where it still fits, its tokens moved)
            for t in range(ctx - (s[i + 1] - s[i]), ctx):
                written[int(tables[i, t // BS]), t % BS] = True
        out = torch.full_like(q, 9.0)
        kvc.kvc_attend(cache_of(x, scales), step, q, out)
        assert torch.equal(out[same], whole[same]) and torch.all(out[~keep] == 9.0)
        y = x.clone()
        kvc.kvc_append(cache_of(y, scales), step, k, k)
        assert torch.equal(y[:, ~written], x[:, ~written])
        back = torch.full_like(k, 9.0)
        kvc.kvc_gather(cache_of(y, scales), step, back, back.clone())
        assert torch.equal(back[keep], k[keep]) and torch.all(back[~keep] == 9.0)


def test_more_rows_than_a_grid_is_wide():
    """2^24 and some rows of eight float32 heads of 128, four waves a token: a step whose last tokens alone have a place (the
    others' context indices are negative), with one row of memory for all of them."""
    N, ctx, heads, d = 17_000_001, 20, 8, 128
    x = torch.zeros(2, 2, BS, heads, d, device=DEV)
    cache = kvc.Cache([x[0]], [x[1]])
    row = torch.randn(2, 1, heads, d, generator=torch.Generator().manual_seed(4)).to(DEV)
    step = kvc.Step([N], [ctx], device=DEV)
    kvc.kvc_append(cache, step, *row.expand(2, N, heads, d))
    flat = x.view(2, 2 * BS, heads, d)
    assert torch.equal(flat[:, :ctx], row.expand(2, ctx, heads, d)) and not torch.any(flat[:, ctx:])


@pytest.mark.parametrize("ctx_bound,kind", [(21760, "f32")])
def test_more_joined_rows_than_a_grid_is_wide(ctx_bound, kind):
    """Seventeen ranges of 2^24 and some rows of heads, a workgroup each in the join: equal sequences get equal results."""
    seqs, new, heads, kv_heads, d = 8200, 32, 64, 8, 64
    N = seqs * new
    assert N * heads > 2 ** 24
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 100 GB: a workspace of 75")
    g = torch.Generator().manual_seed(5)
    x = torch.randn(2, ctx_bound // BS, BS, kv_heads, d, generator=g).to(DEV)
    cache = kvc.Cache([x[0]], [x[1]])
    one = torch.randn(new, heads, d, generator=g).to(DEV)
    step = kvc.Step.on_device(torch.arange(0, N + 1, new, dtype=torch.int32, device=DEV),
                              torch.full((seqs,), new, dtype=torch.int32, device=DEV), N, new, ctx_bound)
    q = one.repeat(seqs, 1, 1)
    assert kvc.kvc_attend_workspace_bytes(cache, step, heads) == 17 * N * heads * (4 * d + 8)
    out = torch.full_like(q, 9.0)
    kvc.kvc_attend(cache, step, q, out)
    want = kvc.kvc_attend(cache, kvc.Step([new], [new], device=DEV), one)
    out = out.view(seqs, new, heads, d)
    assert torch.equal(out, out[:1].expand_as(out))
    # (two orders of the same float32 sums: scores off by 68 2^-24 14, sums over 32 tokens)
    assert torch.all((out[0] - want).abs() <= 2.0 ** -12 * (1 + want.abs()))
    del out, q
    torch.cuda.empty_cache()
