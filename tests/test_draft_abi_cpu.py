"""The entry points of a step of drafted tokens refuse what they do not take, on the host and before any launch.  The
addresses are never dereferenced: each case fails a check, or has no row to work on."""
import ctypes
import math

import pytest
import torch

from paper_2609_34060_amd import kvc

FAKE = 0x7F0000001000
N_, S, D, A, U, W, X = (kvc.KVC_ERR_NULL_ARG, kvc.KVC_ERR_SHAPE, kvc.KVC_ERR_DTYPE, kvc.KVC_ERR_ALIGN,
                        kvc.KVC_ERR_UNSUPPORTED, kvc.KVC_ERR_WORKSPACE, kvc.KVC_ERR_ALIAS)


class Call:
    """What every check accepts, as fake addresses."""

    def __init__(self, dtype=kvc.KVC_BF16, L=2, H=2, d=128, heads=8):
        self.ks, self.vs, self.sk, self.sv = (
            (ctypes.c_void_p * L)(*[FAKE + 0x100000 * (4 * l + j) for l in range(L)]) for j in range(4))
        ptr = lambda a: ctypes.cast(a, ctypes.POINTER(ctypes.c_void_p))
        self.cache = kvc.kvc_cache(dtype, L, H, d, 16, 64, 16 * H * d, H * d, d, ptr(self.ks), ptr(self.vs))
        self.scales = kvc.kvc_scales(ptr(self.sk), ptr(self.sv), 16 * H, 1, 16) if dtype == kvc.KVC_I8 else None
        self.step = kvc.kvc_step(2, 5, 4, 100, 7, 0, FAKE, FAKE + 64, FAKE + 128, FAKE + 256)
        rt = kvc.KVC_F32 if dtype == kvc.KVC_F32 else kvc.KVC_BF16
        self.query = kvc.kvc_query(rt, heads, 1, 0, d ** -0.5, 0, FAKE + 0x30000, heads * d, d, FAKE + 0x40000,
                                   heads * d, d, None)
        self.masks, self.words, self.parents, self.positions = FAKE + 0x50000, 1, FAKE + 0x60000, FAKE + 0x70000
        self.path, self.counts, self.layers, self.layer = FAKE + 0x80000, FAKE + 0x90000, (0, L), 0
        self.ws, self.ws_bytes = FAKE, 1 << 30
        self.freq = (ctypes.c_double * 64)(*[10000.0 ** (-i / 64) for i in range(64)])
        self.rotary = kvc.kvc_rotary(rt, 5, d, kvc.KVC_ROPE_HALF, d, 0, 1.0, ctypes.addressof(self.freq), FAKE)
        self.q = kvc.kvc_heads(heads, 0, FAKE, heads * d, d, FAKE + 0x10000, heads * d, d)
        self.k = kvc.kvc_heads(H, 0, FAKE + 0x20000, H * d, d, FAKE + 0x30000, H * d, d)
        self.draft = kvc.kvc_draft(1000, 0, FAKE, FAKE, FAKE, 1000, FAKE, 1004, FAKE, FAKE, FAKE, FAKE, FAKE)
        self.missing = set()

    def _ref(self, name):
        v = getattr(self, name)
        if v is None or name in self.missing:
            return None
        return bytes(v) if name in ("query", "draft", "rotary", "q", "k") else ctypes.byref(v)

    def tree(self):
        return kvc.load().kvc_tree(self._ref("step"), self.parents, self.masks, self.words, self.positions, None)

    def attend(self):
        return kvc.load().kvc_attend_tree(self._ref("cache"), self._ref("scales"), self._ref("step"), self._ref("query"),
                                          self.masks, self.words, self.layer, self.ws, self.ws_bytes, None)

    def rotate(self):
        return kvc.load().kvc_rotate(self._ref("rotary"), self._ref("q"), self._ref("k"), None)

    def verify(self):
        return kvc.load().kvc_verify(self._ref("step"), self._ref("draft"), self.ws, self.ws_bytes, None)

    def keep(self):
        return kvc.load().kvc_keep(self._ref("cache"), self._ref("scales"), self._ref("step"), self.path, self.counts,
                                   *self.layers, None)


def sets(path, value):
    def change(c):
        obj, _, field = path.rpartition(".")
        setattr(getattr(c, obj) if obj else c, field, value)
    return change


def absent(name):
    return lambda c: c.missing.add(name)


def freq(i, value):
    def change(c):
        c.freq[i] = value
    return change


STEP = [(absent("step"), N_), (sets("step.num_seqs", -1), S), (sets("step.num_rows", -1), S), (sets("step.num_seqs", 0), S),
        (sets("step.max_new", 6), S), (sets("step.max_new", -1), S), (sets("step.max_context", -1), S),
        (sets("step.max_context", (1 << 30) + 1), S), (sets("step.max_blocks", 0), S), (sets("step.reserved", 1), S),
        (sets("step.starts", None), N_), (sets("step.contexts", None), N_), (sets("step.starts", FAKE + 2), A),
        (sets("step.contexts", FAKE + 1), A), (sets("step.offsets", FAKE + 3), A)]
CACHE = [(absent("cache"), N_), (sets("cache.dtype", 3), D), (sets("cache.head_dim", 96), U),
         (sets("cache.num_kv_heads", 0), S), (sets("cache.token_stride", 260), A), (sets("cache.block_stride", 1 << 31), U),
         (sets("cache.k_layers", None), N_), (sets("step.num_rows", 1 << 30), S)]
LONG = [(lambda c: (sets("step.num_rows", 2000)(c), sets("step.max_new", 1025)(c), sets("words", 17)(c)), U)]
TREE = [(sets("parents", None), N_), (sets("masks", None), N_), (sets("parents", FAKE + 2), A), (sets("masks", FAKE + 4), A),
        (sets("positions", FAKE + 1), A), (sets("words", 0), S), (sets("words", -1), S),
        (lambda c: (sets("step.num_rows", 200)(c), sets("step.max_new", 65)(c)), S)]
ATTEND = [(sets("masks", None), N_), (sets("masks", FAKE + 4), A), (sets("words", 0), S), (sets("words", -3), S),
          (lambda c: (sets("step.num_rows", 200)(c), sets("step.max_new", 129)(c), sets("words", 2)(c)), S),
          (sets("query.causal", 0), S), (sets("query.window", 3), U), (sets("query.window", -1), S),
          (absent("query"), N_), (sets("query.dtype", kvc.KVC_F32), D), (sets("query.num_heads", 7), S),
          (sets("query.q", None), N_), (sets("query.out", FAKE + 8), A), (sets("query.scale", math.nan), S),
          (sets("layer", 2), S), (sets("layer", -1), S)]
ROTATE = [(absent("rotary"), N_), (absent("q"), N_), (sets("rotary.dtype", kvc.KVC_I8), D), (sets("rotary.dtype", 7), D),
          (sets("rotary.head_dim", 96), U), (sets("rotary.head_dim", 0), U), (sets("rotary.style", 0), U),
          (sets("rotary.style", 3), U), (sets("rotary.rotary_dim", 0), S), (sets("rotary.rotary_dim", 3), S),
          (sets("rotary.rotary_dim", 130), S), (sets("rotary.rotary_dim", -2), S), (sets("rotary.inverse", 2), S),
          (sets("rotary.inverse", -1), S), (sets("rotary.num_rows", -1), S), (sets("rotary.factor", math.nan), S),
          (sets("rotary.factor", math.inf), S), (sets("rotary.factor", 65537.0), S), (sets("rotary.inv_freq", None), N_),
          (freq(63, math.nan), S), (freq(0, -math.inf), S), (freq(5, 1e6), S), (sets("rotary.positions", None), N_),
          (sets("rotary.positions", FAKE + 2), A), (sets("q.reserved", 1), S), (sets("k.num_heads", -1), S),
          (sets("q.num_heads", 65536), S), (sets("q.in_", None), N_), (sets("k.out", None), N_), (sets("q.in_", FAKE + 8), A),
          (sets("k.out", FAKE + 4), A), (sets("q.in_token_stride", 1028), A), (sets("q.in_head_stride", 130), A),
          (sets("k.out_token_stride", 257), A), (sets("k.out_head_stride", 132), A), (sets("q.in_token_stride", -1024), S),
          (sets("q.out_head_stride", 64), S), (sets("q.out_token_stride", 0), S), (sets("k.in_head_stride", 1 << 41), S),
          (lambda c: (sets("q.out", FAKE)(c), sets("q.in_token_stride", 2048)(c)), X),
          (lambda c: (sets("q.out", FAKE)(c), sets("q.in_head_stride", 256)(c)), X)]
VERIFY = [(absent("draft"), N_), (sets("draft.vocab", 0), S), (sets("draft.vocab", (1 << 30) + 1), S),
          (sets("draft.children", -1), S), (sets("draft.target_stride", 999), S), (sets("draft.draft_stride", 10), S),
          (sets("draft.target_stride", 1 << 41), S),
          *[(sets("draft." + x, None), N_) for x in ("parents", "tokens", "target", "uniforms", "last", "path", "counts",
                                                     "chosen")],
          *[(sets("draft." + x, FAKE + 2), A) for x in ("parents", "tokens", "target", "draft", "uniforms", "last", "path",
                                                        "counts", "chosen")],
          (sets("ws", None), W), (sets("ws", FAKE + 128), W), (sets("ws_bytes", 256 + 2 * 16 - 1), W), (sets("ws_bytes", 0), W)]
KEEP = [(sets("path", None), N_), (sets("counts", None), N_), (sets("path", FAKE + 1), A), (sets("counts", FAKE + 2), A),
        (sets("layers", (0, 3)), S), (sets("layers", (1, 0)), S), (sets("layers", (-1, 1)), S)]
SCALED = [(absent("scales"), N_), (sets("scales.k_layers", None), N_), (sets("scales.token_stride", 0), S)]

CASES = ([(call, kvc.KVC_BF16, *x) for call in ("tree", "attend", "verify", "keep") for x in STEP] +
         [(call, kvc.KVC_BF16, *x) for call in ("attend", "keep") for x in CACHE] +
         [(call, kvc.KVC_I8, *x) for call in ("attend", "keep") for x in SCALED] +
         [(call, kvc.KVC_BF16, *x) for call, xs in (("tree", TREE + LONG), ("attend", ATTEND), ("rotate", ROTATE),
                                                   ("verify", VERIFY + LONG), ("keep", KEEP)) for x in xs])


@pytest.mark.parametrize("at", range(len(CASES)))
def test_refused(at):
    call, dtype, change, status = CASES[at]
    c = Call(dtype)
    change(c)
    assert getattr(c, call)() == status


def test_nothing_to_do():
    """Steps and rows of nothing are taken, before any pointer that they do not need is asked for."""
    c = Call()
    c.step.num_rows = c.step.max_new = 0
    c.parents = c.masks = c.path = c.counts = None
    assert c.tree() == c.attend() == c.keep() == kvc.KVC_OK
    c.step.num_seqs = 0
    c.draft.counts = None
    assert c.verify() == kvc.KVC_OK
    c.rotary.num_rows = 0
    c.rotary.positions = None
    assert c.rotate() == kvc.KVC_OK
    c = Call()
    c.layers = (1, 1)
    assert c.keep() == kvc.KVC_OK
    c.q.num_heads = 0
    c.missing.add("k")
    assert c.rotate() == kvc.KVC_OK


@pytest.mark.parametrize("window", [0, 1 << 19, (1 << 31) - 1])
def test_windows_of_masks(window):
    """Long windows are taken; a workspace that is missing shows that the call came so far."""
    c = Call()
    c.step.max_context, c.ws_bytes, c.step.max_blocks, c.query.window = 1 << 20, 0, 1 << 16, window
    assert c.attend() == W


@pytest.mark.parametrize("n,vocab", [(1, 1), (1, 2048), (3, 2049), (64, 131072), (1000, 50021)])
def test_verify_workspace(n, vocab):
    """A piece of 2048 probabilities leaves two sums, a sequence where it ended."""
    step = kvc.kvc_step(n, n, 1, 10, 0, 0, FAKE, FAKE, None, None)
    need = kvc.load().kvc_verify_workspace_bytes(ctypes.addressof(step), vocab)
    assert n * (16 * -(-vocab // 2048) + 24) <= need <= n * (16 * -(-vocab // 2048) + 32) + 256
    assert kvc.load().kvc_verify_workspace_bytes(ctypes.addressof(step), 0) == 0
    assert kvc.load().kvc_verify_workspace_bytes(None, vocab) == 0


def test_frequencies():
    """theta^(-2 i / r); all slowed, or by the turns over the trained context; the factor."""
    f = kvc.rope_frequencies(128, 500000.0)
    assert len(f) == 64 and f[0] == 1.0 and math.isclose(f[32], 500000.0 ** -0.5, rel_tol=1e-15)
    assert all(math.isclose(a, b / 4, rel_tol=1e-15) for a, b in zip(kvc.rope_frequencies(128, 500000.0, 4.0), f))
    g = kvc.rope_frequencies(128, 500000.0, 8.0, trained=8192)
    turns = [8192 * x / (2 * math.pi) for x in f]
    for a, b, t in zip(g, f, turns):
        k = 1.0 if t >= 32 else 0.0 if t <= 1 else (t - 1) / 31
        assert math.isclose(a, b * k + b / 8 * (1 - k), rel_tol=1e-14)
    assert kvc.rope_factor(1.0) == kvc.rope_factor(0.5) == 1.0 and math.isclose(kvc.rope_factor(8.0), 1 + 0.1 * math.log(8))
    for bad in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=8, theta=0.0), dict(rotary_dim=8, scale=-1.0),
                dict(rotary_dim=8, scale=2.0, trained=100, slow=3.0, fast=3.0)):
        with pytest.raises(ValueError):
            kvc.rope_frequencies(**bad)


def test_python_refusals():
    """Shapes, types and layouts that the binding refuses before the library is asked."""
    step = kvc.Step([2, 1], [5, 3], device="cpu")
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError, match="parents"):
        kvc.kvc_tree(step, i(4))
    with pytest.raises(ValueError, match="parents"):
        kvc.kvc_tree(step, torch.zeros(3))
    with pytest.raises(ValueError, match="parents"):
        kvc.kvc_tree(step, i(6)[::2])
    with pytest.raises(ValueError, match="GPU"):
        kvc.kvc_tree(step, i(3))
    rot = kvc.Rotary(kvc.rope_frequencies(64), 64)
    x = torch.zeros(3, 2, 64)
    for args in ((x[0],), (x[..., :32],), (x.half(),), (x, x[:2]), (x, x.bfloat16()), (x, None, x[:1]),
                 (x, x, None, x.bfloat16())):
        with pytest.raises(ValueError):
            kvc.kvc_rotate(rot, i(3), *args)
    with pytest.raises(ValueError, match="k_out"):
        kvc.kvc_rotate(rot, i(3), x, None, None, x)
    with pytest.raises(ValueError, match="positions"):
        kvc.kvc_rotate(rot, i(2), x)
    with pytest.raises(ValueError, match="positions"):
        kvc.kvc_rotate(rot, torch.zeros(3, dtype=torch.int64), x)
    with pytest.raises(ValueError, match="GPU"):
        kvc.kvc_rotate(rot, i(3), x)
    with pytest.raises(ValueError, match="GPU"):
        kvc.kvc_verify(step, i(3), i(3), torch.zeros(3, 7), torch.zeros(3), torch.zeros(2))
    pool = torch.zeros(4, 16, 2, 64)
    cache = kvc.Cache([pool], [pool])
    with pytest.raises(ValueError, match="GPU"):
        kvc.kvc_keep(cache, step, i(3), i(2))
    with pytest.raises(ValueError, match="masks"):
        kvc.kvc_attend_tree(cache, step, torch.zeros(3, dtype=torch.int64), x)
    with pytest.raises(ValueError, match="masks"):
        kvc.kvc_attend_tree(cache, step, torch.zeros(2, 1, dtype=torch.int64), x)
