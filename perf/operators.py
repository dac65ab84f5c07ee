"""Performance cases of a served step over the paged cache: writing the new tokens (`append`), reading rows back
(`gather`) and the attention of the new tokens over their contexts (`attend`).

A step holds n sequences.  Sequence i has q_i new tokens, rows starts[i] .. starts[i + 1] - 1 of the token-major arrays
[N, heads, head_dim], and c_i tokens in the cache, the new ones among them (its last q_i); its token t sits at position
offset_i + t of its block sequence.  A cache holds float32, bfloat16 or int8 rows; an int8 row (one token, one head, K
or V) has a float32 scale: scale = max|x| / 127, code = rint(x * (127 / max|x|)), value = code * scale.

  append   the new rows are written into the cache; from an int8 cache they are read back as well, so that what was
           kept comes out as the values that it stands for.
  gather   rows of the cache are read into dense arrays.
  attend   out = softmax(scale q K^T) V over the tokens that a query may see, and the log-sum-exp of its scores.

With `own` false the operators are computed by elementary torch operations in float32, else by the package's kernels.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"


def _case(name, op, **kw):
    c = {"name": name, "op": op, "layers": 1, "heads": 8, "q_heads": 32, "dim": 128, "cache": "bf16", "rows": "bf16",
         "block": 16, "seqs": 1, "new_min": 1, "new_max": 1, "ctx_min": 1, "ctx_max": 1, "causal": True, "window": 0,
         "offset": 0}
    c.update(kw)
    return c


def listed():
    return [
        # One decode step's new tokens of 64 requests written into an int8 cache and read back: latency.
        _case("append_decode_i8", "append", cache="i8", seqs=64, ctx_min=1024, ctx_max=16384),
        # A 4K shared segment of an 8B model, all layers, packed into an int8 cache after its prefill or correction.
        _case("append_segment_i8", "append", layers=32, cache="i8", new_min=4096, new_max=4096, ctx_min=4096,
              ctx_max=4096),
        # A short float32 context (the "tiny" workload's heads) read back from an int8 cache, odd lengths: latency.
        _case("gather_tiny_i8", "gather", layers=2, heads=4, dim=64, cache="i8", rows="f32", seqs=3, new_min=17,
              new_max=257, ctx_min=257, ctx_max=300, block=24, offset=5),
        # Whole contexts of eight requests read back for a fit: four layers, bf16 rows from an int8 cache.
        _case("gather_contexts_i8", "gather", layers=4, cache="i8", seqs=8, new_min=1024, new_max=8191, ctx_min=8192,
              ctx_max=8192),
        # The smallest attention: one new token of one request with a short context.
        _case("attend_decode_one", "attend", ctx_min=1000, ctx_max=1000),
        # A decode step of the serving batch: 64 requests, contexts of 1K-16K tokens.
        _case("attend_decode_batch", "attend", seqs=64, ctx_min=1024, ctx_max=16384),
        # The same over an int8 cache, half of the bytes.
        _case("attend_decode_batch_i8", "attend", cache="i8", seqs=64, ctx_min=1024, ctx_max=16384),
        # One request at the end of a 32K context, seven query heads for each of four KV heads: few rows, a long axis.
        _case("attend_decode_long", "attend", heads=4, q_heads=28, ctx_min=32771, ctx_max=32771),
        # The prefill of an ordinary context.
        _case("attend_prefill_4k", "attend", new_min=4096, new_max=4096, ctx_min=4096, ctx_max=4096),
        # A chunk of 2K new tokens at the end of a 32K context that is held in 8 bits: the largest.
        _case("attend_chunk_32k_i8", "attend", cache="i8", new_min=2048, new_max=2048, ctx_min=32768, ctx_max=32768),
        # A mixed step, chunks beside single tokens, with a sliding window and ragged lengths.
        _case("attend_mixed_window", "attend", heads=4, q_heads=28, seqs=16, new_min=1, new_max=509, ctx_min=700,
              ctx_max=8000, window=1024, offset=3),
        # Float32 rows of the "tiny" workload: short chunks and odd lengths.
        _case("attend_tiny_f32", "attend", heads=4, q_heads=4, dim=64, cache="f32", rows="f32", seqs=3, new_min=1,
              new_max=257, ctx_min=129, ctx_max=257),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choices(["append", "gather", "attend"], [25, 15, 60])[0]
    c = _case("", op)
    del c["name"]
    c["heads"], c["q_heads"], c["dim"] = rng.choice([(8, 32, 128), (8, 32, 128), (4, 28, 128), (8, 64, 128), (4, 4, 64),
                                                     (8, 40, 128), (2, 16, 128), (8, 32, 64)])
    c["cache"] = rng.choices(["bf16", "i8", "f32"], [45, 40, 15])[0]
    if op != "attend":
        c["cache"] = rng.choices(["i8", "bf16", "f32"], [70, 20, 10])[0]
        c["q_heads"] = c["heads"]
        c["layers"] = log_int(1, 32)
    c["rows"] = "f32" if c["cache"] == "f32" or (c["cache"] == "i8" and op != "attend" and rng.random() < 0.25) else "bf16"
    c["block"] = rng.choice([16, 16, 16, 8, 32, 64, 24])
    c["offset"] = rng.choice([0, 0, rng.randrange(0, 4 * c["block"])])
    c["seqs"] = rng.choice([1, 1, 2, 3, log_int(2, 16), log_int(8, 64), 64])
    c["ctx_max"] = log_int(16, 32768)
    c["ctx_min"] = max(1, int(c["ctx_max"] * rng.uniform(0.05, 1.0)))
    c["new_max"] = rng.choice([1, 1, rng.randrange(2, 9), log_int(2, 4096), c["ctx_min"]])
    c["new_max"] = min(c["new_max"], c["ctx_min"], 8192)
    c["new_min"] = c["new_max"] if c["seqs"] == 1 else rng.choice([c["new_max"], max(1, c["new_max"] // 4), 1])
    if op == "attend":
        c["causal"] = rng.random() < 0.9
        if c["causal"] and rng.random() < 0.2:
            c["window"] = log_int(16, 4096)

    def too_large():
        # no drawn case costs more than the largest listed one, nor holds more of the plain form's scores
        w = work(c)
        pools = 2.0 * c["layers"] * c["seqs"] * c["ctx_max"] * c["heads"] * c["dim"] * _es(c["cache"])
        if op != "attend":
            return w["bytes"] > 1.3e9 or pools > 2.5e9
        scores = c["seqs"] * c["q_heads"] * c["new_max"] * c["ctx_max"]
        return (w["bytes"] > 2.2e9 or w["flops"] > (1.0e12 if c["cache"] != "f32" else 1e11) or scores > 2.1e9
                or c["seqs"] * c["ctx_max"] * c["heads"] * c["dim"] > 1.1e9)

    while too_large():
        if c["layers"] > 1:
            c["layers"] = (c["layers"] + 1) // 2
        elif c["seqs"] > 4:
            c["seqs"] = (c["seqs"] * 2 + 1) // 3
        else:
            c["ctx_max"] = c["ctx_max"] * 3 // 4 + 1
            c["ctx_min"] = min(c["ctx_min"], c["ctx_max"])
            c["new_max"] = max(1, min(c["new_max"] * 4 // 5, c["ctx_min"]))
            c["new_min"] = min(c["new_min"], c["new_max"])
            if c["seqs"] == 1:
                c["new_min"] = c["new_max"]
    return c


# ---- sizes -----------------------------------------------------------------------------------------------------

def _lengths(c):
    """New tokens and contexts of the sequences: uniform in their ranges, new tokens on a logarithm's scale."""
    rng = np.random.Generator(np.random.PCG64([77, c["seqs"], c["ctx_max"], c["new_max"]]))
    ctx = rng.integers(c["ctx_min"], c["ctx_max"] + 1, size=c["seqs"])
    new = np.exp(rng.uniform(math.log(c["new_min"]), math.log(c["new_max"] + 1), size=c["seqs"])).astype(np.int64)
    new = np.minimum(np.clip(new, c["new_min"], c["new_max"]), ctx)
    return new, ctx.astype(np.int64)


def _es(name):
    return {"f32": 4, "bf16": 2, "i8": 1}[name]


def _dt(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.int8}[name]


def work(case):
    c = case
    new, ctx = _lengths(c)
    H, d, N = c["heads"], c["dim"], int(new.sum())
    held = d * _es(c["cache"]) + (4 if c["cache"] == "i8" else 0)  # one row of the cache
    row = d * _es(c["rows"])
    if c["op"] == "append":
        rows = 2 * c["layers"] * N * H
        back = row if c["cache"] == "i8" else 0
        return {"bytes": float(rows * (row + held + back)), "flops": float(rows * d * 3)}
    if c["op"] == "gather":
        rows = 2 * c["layers"] * N * H
        return {"bytes": float(rows * (row + held)), "flops": float(rows * d)}
    pairs = read = 0
    for q, n in zip(new.tolist(), ctx.tolist()):
        pos = np.arange(n - q, n, dtype=np.int64)
        hi = pos + 1 if c["causal"] else np.full(q, n, dtype=np.int64)
        lo = np.maximum(0, pos + 1 - c["window"]) if c["window"] else np.zeros(q, dtype=np.int64)
        pairs += int((hi - lo).sum())
        read += int(hi.max() - lo.min())
    Hq = c["q_heads"]
    return {"bytes": float(2 * read * H * held + N * Hq * (2 * row + 4)), "flops": float(4 * d * pairs * Hq)}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _normal(g, shape, dtype):
    """N(0, 1) rows; four feature channels are three times as wide, as the keys' channels of a trained model are."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)
    x[..., 3::shape[-1] // 4] *= 3.0
    return x.to(dtype)


def _fill(g, pools, scales, dtype):
    for i in range(pools.shape[0]):
        x = _normal(g, tuple(pools.shape[1:]), torch.float32)
        if scales is None:
            pools[i] = x.to(dtype)
        else:
            top = x.abs().amax(-1)
            most = torch.full_like(top, 127.0)  # (a division by a tensor is a division; one by a number need not be)
            pools[i] = torch.round(x * (most / top)[..., None]).to(torch.int8)
            scales[i] = top / most


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(np.random.SeedSequence([int(seed), c["seqs"], c["ctx_max"], c["dim"]]).generate_state(1)[0]))
    new, ctx = _lengths(c)
    n, N, H, d, bs, L = c["seqs"], int(new.sum()), c["heads"], c["dim"], c["block"], c["layers"]
    off = np.array([c["offset"] * (i % 3) // 2 for i in range(n)], dtype=np.int64)
    blocks = -(-(off + ctx) // bs)
    nb = int(blocks.sum()) + 3
    order = torch.randperm(nb, generator=g, device=DEV).to(torch.int32)
    # every sequence owns its blocks, scattered over the pool
    tables = torch.zeros(n, int(blocks.max()), dtype=torch.int32, device=DEV)
    at = 0
    for i in range(n):
        tables[i, : blocks[i]] = order[at: at + int(blocks[i])]
        at += int(blocks[i])

    def device(v):
        return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)

    pools = torch.empty(2 * L, nb, bs, H, d, dtype=_dt(c["cache"]), device=DEV)  # K of every layer, then V
    scales = None
    if c["cache"] == "i8":  # a block's scales lie head by head, [block, slot, head] being a view of them
        scales = torch.empty(2 * L, nb, H, bs, dtype=torch.float32, device=DEV).permute(0, 1, 3, 2)
    if c["op"] == "append":
        pools.zero_()
        if scales is not None:
            scales.zero_()
    else:
        _fill(g, pools, scales, _dt(c["cache"]))
    st = {"c": c, "n": n, "N": N, "max_new": int(new.max()), "max_ctx": int(ctx.max()), "tables": tables,
          "starts": device(np.concatenate([[0], np.cumsum(new)])), "contexts": device(ctx), "offsets": device(off),
          "pools": pools, "scales": scales}
    if c["op"] == "attend":
        st["q"] = _normal(g, (N, c["q_heads"], d), _dt(c["rows"]))
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(N, c["q_heads"], dtype=torch.float32, device=DEV)
    else:
        st["k"], st["v"] = (torch.empty(L, N, H, d, dtype=_dt(c["rows"]), device=DEV) for _ in range(2))
        if c["op"] == "append":
            for x in (st["k"], st["v"]):
                for i in range(L):
                    x[i] = _normal(g, (N, H, d), x.dtype)
            st["back_k"], st["back_v"] = torch.empty_like(st["k"]), torch.empty_like(st["v"])
    if own:  # the handles that a serving program holds: its cache, and the step that all layers of a model share
        from paper_2609_34060_amd import kvc
        st["cache"] = kvc.Cache(list(pools[:L]), list(pools[L:]),
                                k_scales=None if scales is None else list(scales[:L]),
                                v_scales=None if scales is None else list(scales[L:]))
        st["step"] = kvc.Step(new.tolist(), ctx.tolist(), tables, offsets=off.tolist())
        if c["op"] == "attend":
            need = kvc.kvc_attend_workspace_bytes(st["cache"], st["step"], c["q_heads"])
            st["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
    return st


# ---- the plain form --------------------------------------------------------------------------------------------

def _token_places(st):
    """Block and slot of every new token, with its sequence and its place among the sequence's new tokens."""
    row = torch.arange(st["N"], device=DEV)
    starts = st["starts"].long()
    seq = torch.searchsorted(starts, row, right=True) - 1
    j = row - starts[seq]
    new = starts[1:] - starts[:-1]
    p = (st["offsets"].long() + st["contexts"].long() - new)[seq] + j
    bs = st["c"]["block"]
    return st["tables"][seq, p // bs].long(), p % bs, seq, j


def _plain_append(st):
    c, L = st["c"], st["c"]["layers"]
    blk, slot, _, _ = _token_places(st)
    x = torch.cat([st["k"], st["v"]])
    if st["scales"] is None:
        st["pools"][:, blk, slot] = x
        return {"pools": st["pools"]}
    x = x.float()
    top = x.abs().amax(-1)
    most = torch.full_like(top, 127.0)
    codes = torch.round(x * (most / top)[..., None])
    st["pools"][:, blk, slot] = codes.to(torch.int8)
    st["scales"][:, blk, slot] = top / most
    back = st["pools"][:, blk, slot].float() * st["scales"][:, blk, slot][..., None]
    back = back.to(_dt(c["rows"]))
    return {"k": back[:L], "v": back[L:], "scales": st["scales"]}


def _plain_gather(st):
    c, L = st["c"], st["c"]["layers"]
    blk, slot, _, _ = _token_places(st)
    x = st["pools"][:, blk, slot]
    if st["scales"] is not None:
        x = x.float() * st["scales"][:, blk, slot][..., None]
    x = x.to(_dt(c["rows"]))
    return {"k": x[:L], "v": x[L:]}


def _plain_attend(st):
    c = st["c"]
    n, Q, T, H, d, bs = st["n"], st["max_new"], st["max_ctx"], c["heads"], c["dim"], c["block"]
    G = c["q_heads"] // H
    _, _, seq, j = _token_places(st)
    ctx, starts = st["contexts"].long(), st["starts"].long()
    new = starts[1:] - starts[:-1]
    t = torch.arange(T, device=DEV)
    p = st["offsets"].long()[:, None] + t
    there = t < ctx[:, None]  # [n, T]
    blk = st["tables"].gather(1, (p // bs).clamp(max=st["tables"].shape[1] - 1)).long()
    k, v = (st["pools"][i][blk, p % bs].float() for i in (0, 1))  # [n, T, H, d]
    if st["scales"] is not None:
        k *= st["scales"][0][blk, p % bs][..., None]
        v *= st["scales"][1][blk, p % bs][..., None]
    v = torch.where(there[..., None, None], v, 0.0)
    rows = (starts[:-1, None] + torch.arange(Q, device=DEV)).clamp(max=st["N"] - 1)
    q = st["q"][rows].float().reshape(n, Q, H, G, d).permute(0, 2, 1, 3, 4).reshape(n, H, Q * G, d)
    s = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous())  # [n, H, Q G, T]
    s *= 1.0 / math.sqrt(d)
    pos = (ctx - new)[:, None] + torch.arange(Q, device=DEV)  # [n, Q]
    see = there[:, None, :] if not c["causal"] else there[:, None, :] & (t <= pos[..., None])
    if c["window"]:
        see = see & (t > pos[..., None] - c["window"])
    see = see.expand(n, Q, T).repeat_interleave(G, dim=1)[:, None]
    s.masked_fill_(~see, -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    s -= m
    s.exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s, v.permute(0, 2, 1, 3).contiguous()) / total.clamp(min=1e-38)
    lse = (m + total.log())[..., 0].reshape(n, H, Q, G)
    out = o.reshape(n, H, Q, G, d)[seq, :, j].reshape(st["N"], c["q_heads"], d).to(_dt(c["rows"]))
    return {"out": out, "lse": lse[seq, :, j].reshape(st["N"], c["q_heads"])}


def run(state):
    st = state
    op = st["c"]["op"]
    if not own:
        return {"append": _plain_append, "gather": _plain_gather, "attend": _plain_attend}[op](st)
    from paper_2609_34060_amd import kvc
    if op == "attend":
        kvc.kvc_attend(st["cache"], st["step"], st["q"], st["out"], lse=st["lse"], causal=st["c"]["causal"],
                       window=st["c"]["window"], workspace=st["workspace"])
        return {"out": st["out"], "lse": st["lse"]}
    if op == "gather":
        kvc.kvc_gather(st["cache"], st["step"], st["k"], st["v"])
        return {"k": st["k"], "v": st["v"]}
    kvc.kvc_append(st["cache"], st["step"], st["k"], st["v"])
    if st["scales"] is None:
        return {"pools": st["pools"]}
    kvc.kvc_gather(st["cache"], st["step"], st["back_k"], st["back_v"])
    return {"k": st["back_k"], "v": st["back_v"], "scales": st["scales"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    c, st = case, prepare(case, seed)
    new, ctx = _lengths(c)
    tables, off = st["tables"].cpu().numpy(), st["offsets"].cpu().numpy()
    L, H, d, bs = c["layers"], c["heads"], c["dim"], c["block"]

    def places(i, first, last):
        p = np.arange(first, last) + off[i]
        return torch.from_numpy(tables[i, p // bs]).long().to(DEV), torch.from_numpy(p % bs).long().to(DEV)

    def held(pool, scale, b, s):
        x = pool[b, s].to(torch.float64)
        return x if scale is None else x * scale[b, s].to(torch.float64).unsqueeze(-1)

    ends = np.cumsum(new)
    if c["op"] == "attend":
        G = c["q_heads"] // H
        out = torch.empty(st["N"], c["q_heads"], d, dtype=torch.float64, device=DEV)
        lse = torch.empty(st["N"], c["q_heads"], dtype=torch.float64, device=DEV)
        for i in range(c["seqs"]):
            q_n, T = int(new[i]), int(ctx[i])
            a, z = int(ends[i]) - q_n, int(ends[i])
            b, s = places(i, 0, T)
            ks = held(st["pools"][0], None if st["scales"] is None else st["scales"][0], b, s)
            vs = held(st["pools"][1], None if st["scales"] is None else st["scales"][1], b, s)
            key, query = torch.arange(T, device=DEV)[None], torch.arange(T - q_n, T, device=DEV)[:, None]
            hidden = torch.zeros(q_n, T, dtype=torch.bool, device=DEV)
            if c["causal"]:
                hidden |= key > query
            if c["window"]:
                hidden |= query - key >= c["window"]
            for h in range(c["q_heads"]):
                z_ = st["q"][a:z, h].to(torch.float64) @ ks[:, h // G].T / math.sqrt(d)
                z_[hidden] = -math.inf
                top = torch.logsumexp(z_, 1)
                lse[a:z, h] = top
                out[a:z, h] = torch.exp(z_ - top[:, None]) @ vs[:, h // G]
        return {"out": out, "lse": lse}
    if c["op"] == "append" and st["scales"] is None:
        pools = st["pools"].to(torch.float64)
    res = [torch.empty(L, st["N"], H, d, dtype=torch.float64, device=DEV) for _ in range(2)]
    scales = None if st["scales"] is None else st["scales"].to(torch.float64)
    for i in range(c["seqs"]):
        a, z = int(ends[i] - new[i]), int(ends[i])
        b, s = places(i, int(ctx[i] - new[i]), int(ctx[i]))
        for kv in range(2):
            for l in range(L):
                u = kv * L + l
                if c["op"] == "gather":
                    res[kv][l, a:z] = held(st["pools"][u], None if scales is None else st["scales"][u], b, s)
                    continue
                x = (st["k"], st["v"])[kv][l, a:z].to(torch.float64)
                if scales is None:
                    pools[u][b, s] = x
                    continue
                step = x.abs().amax(-1) / 127
                scales[u][b, s] = step
                res[kv][l, a:z] = torch.round(x / step[..., None]) * step[..., None]
    if c["op"] == "gather":
        return {"k": res[0], "v": res[1]}
    return {"pools": pools} if scales is None else {"k": res[0], "v": res[1], "scales": scales}
