"""The served step's entry points refuse what they do not take, on the host and before any launch.  The addresses are
never dereferenced: each case fails a check, or has no row to work on."""
import ctypes

import pytest
import torch

from paper_2609_34060_amd import kvc

FAKE = 0x7F0000001000
BIG = 1 << 31


class Call:
    """A cache, a step, rows and a query that every check accepts, as fake addresses."""

    def __init__(self, dtype=kvc.KVC_BF16, L=2, H=2, d=128, bs=16, nb=64, N=5, n=2, heads=8):
        self.ks, self.vs, self.sk, self.sv = (
            (ctypes.c_void_p * L)(*[FAKE + 0x100000 * (4 * l + j) for l in range(L)]) for j in range(4))
        ptr = lambda a: ctypes.cast(a, ctypes.POINTER(ctypes.c_void_p))
        self.cache = kvc.kvc_cache(dtype, L, H, d, bs, nb, bs * H * d, H * d, d, ptr(self.ks), ptr(self.vs))
        self.scales = kvc.kvc_scales(ptr(self.sk), ptr(self.sv), bs * H, 1, bs) if dtype == kvc.KVC_I8 else None
        self.step = kvc.kvc_step(n, N, 4, 100, 7, 0, FAKE, FAKE + 64, FAKE + 128, FAKE + 256)
        rt = kvc.KVC_F32 if dtype == kvc.KVC_F32 else kvc.KVC_BF16
        self.rows = kvc.kvc_rows(rt, 0, FAKE + 0x10000, FAKE + 0x20000, N * H * d, H * d, d)
        self.query = kvc.kvc_query(rt, heads, 1, 0, d ** -0.5, 0, FAKE + 0x30000, heads * d, d, FAKE + 0x40000,
                                   heads * d, d, None)
        self.layers, self.layer, self.ws, self.ws_bytes = (0, L), 0, FAKE, 1 << 30
        self.missing = set()

    def _ref(self, name):
        v = getattr(self, name)
        if v is None or name in self.missing:
            return None
        return bytes(v) if name in ("rows", "query") else ctypes.byref(v)  # (as the binding passes them)

    def append(self, gather=False):
        f = kvc.load().kvc_gather if gather else kvc.load().kvc_append
        return f(self._ref("cache"), self._ref("scales"), self._ref("step"), self._ref("rows"), *self.layers, None)

    def gather(self):
        return self.append(gather=True)

    def attend(self):
        return kvc.load().kvc_attend(self._ref("cache"), self._ref("scales"), self._ref("step"), self._ref("query"),
                                     self.layer, self.ws, self.ws_bytes, None)


def setter(path, value):
    def change(c):
        obj, _, field = path.rpartition(".")
        setattr(getattr(c, obj) if obj else c, field, value)
    return change


def pointer(array, at, value):
    def change(c):
        getattr(c, array)[at] = value
    return change


def absent(name):
    return lambda c: c.missing.add(name)


N, S, D, A, U, W = (kvc.KVC_ERR_NULL_ARG, kvc.KVC_ERR_SHAPE, kvc.KVC_ERR_DTYPE, kvc.KVC_ERR_ALIGN,
                    kvc.KVC_ERR_UNSUPPORTED, kvc.KVC_ERR_WORKSPACE)
# what every one of the three refuses (the cache and the step)
SHARED = [
    (absent("cache"), N), (absent("step"), N), (setter("cache.dtype", 3), D), (setter("cache.head_dim", 96), U),
    (setter("cache.head_dim", 256), U), (setter("cache.num_kv_heads", 0), S), (setter("cache.num_kv_heads", 65536), S),
    (setter("cache.block_size", 0), S), (setter("cache.num_blocks", 0), S), (setter("cache.token_stride", 0), S),
    (setter("cache.block_stride", -64), S), (setter("cache.head_stride", 64), S), (setter("cache.token_stride", 260), A),
    (setter("cache.block_stride", 4100), A), (setter("cache.head_stride", 132), A),
    (setter("cache.block_stride", BIG), U), (setter("cache.token_stride", BIG), U),
    (setter("cache.k_layers", None), N), (setter("cache.v_layers", None), N),
    (pointer("ks", 0, None), N), (pointer("vs", 0, FAKE + 8), A),
    (setter("step.num_seqs", -1), S), (setter("step.num_seqs", (1 << 30) + 1), S), (setter("step.num_rows", -1), S),
    (setter("step.num_seqs", 0), S),
    (setter("step.max_new", 6), S), (setter("step.max_new", -1), S), (setter("step.max_context", -1), S),
    (setter("step.max_context", (1 << 30) + 1), S), (setter("step.max_blocks", -1), S),
    (setter("step.max_blocks", 0), S), (setter("step.reserved", 1), S), (setter("step.num_rows", 1 << 30), S),
    (setter("step.starts", None), N), (setter("step.contexts", None), N), (setter("step.starts", FAKE + 2), A),
    (setter("step.contexts", FAKE + 1), A), (setter("step.offsets", FAKE + 3), A), (setter("step.tables", FAKE + 2), A),
]
SCALED = [
    (absent("scales"), N), (setter("scales.k_layers", None), N), (setter("scales.v_layers", None), N),
    (pointer("sk", 0, None), N), (pointer("sv", 0, FAKE + 2), A), (setter("scales.block_stride", 0), S),
    (setter("scales.token_stride", -1), S), (setter("scales.head_stride", 0), S),
    (setter("scales.block_stride", 1 << 30), U), (setter("scales.token_stride", 1 << 30), U),
    (setter("cache.token_stride", 264), A), (setter("cache.block_stride", 1 << 32), U),
]
MOVES = [
    (absent("rows"), N), (setter("rows.reserved", 1), S), (setter("rows.dtype", kvc.KVC_I8), D),
    (setter("rows.dtype", 9), D), (setter("rows.dtype", kvc.KVC_F32), D), (setter("rows.k", None), N),
    (setter("rows.v", None), N), (setter("rows.k", FAKE + 8), A), (setter("rows.v", FAKE + 2), A),
    (setter("rows.token_stride", 260), A), (setter("rows.head_stride", 132), A), (setter("rows.layer_stride", 4), A),
    (setter("rows.token_stride", -256), S), (setter("rows.head_stride", -128), S),
    (setter("rows.layer_stride", -1280), S), (setter("layers", (0, 3)), S), (setter("layers", (2, 1)), S),
    (setter("layers", (-1, 1)), S),
]
ATTEND = [
    (absent("query"), N), (setter("query.reserved", 1), S), (setter("query.causal", 2), S),
    (setter("query.causal", -1), S), (setter("query.window", -1), S), (setter("query.scale", float("nan")), S),
    (setter("query.scale", float("inf")), S), (setter("query.dtype", kvc.KVC_F32), D),
    (setter("query.dtype", kvc.KVC_I8), D), (setter("query.num_heads", 0), S), (setter("query.num_heads", 7), S),
    (setter("query.num_heads", 1 << 30), S), (setter("query.q", None), N), (setter("query.out", None), N),
    (setter("query.q", FAKE + 8), A), (setter("query.out", FAKE + 4), A), (setter("query.lse", FAKE + 2), A),
    (setter("query.q_token_stride", 1028), A), (setter("query.q_head_stride", 130), A),
    (setter("query.out_token_stride", 1025), A), (setter("query.out_head_stride", 4), A),
    (setter("query.q_token_stride", -1024), S), (setter("query.q_head_stride", -128), S),
    (setter("query.out_token_stride", -1024), S), (setter("query.out_head_stride", -128), S),
    (setter("layer", -1), S), (setter("layer", 2), S),
]


@pytest.mark.parametrize("call", ["append", "gather", "attend"])
@pytest.mark.parametrize("at", range(len(SHARED)))
def test_cache_and_step(call, at):
    change, status = SHARED[at]
    c = Call()
    change(c)
    assert getattr(c, call)() == status


@pytest.mark.parametrize("call", ["append", "gather", "attend"])
@pytest.mark.parametrize("at", range(len(SCALED)))
def test_scales(call, at):
    change, status = SCALED[at]
    c = Call(dtype=kvc.KVC_I8)
    change(c)
    assert getattr(c, call)() == status


@pytest.mark.parametrize("call", ["append", "gather"])
@pytest.mark.parametrize("at", range(len(MOVES)))
def test_rows(call, at):
    change, status = MOVES[at]
    c = Call()
    change(c)
    assert getattr(c, call)() == status


@pytest.mark.parametrize("at", range(len(ATTEND)))
def test_queries(at):
    change, status = ATTEND[at]
    c = Call()
    change(c)
    assert c.attend() == status


@pytest.mark.parametrize("call", ["append", "gather", "attend"])
def test_scales_go_with_8_bit_caches_only(call):
    c = Call()
    c.scales = Call(dtype=kvc.KVC_I8).scales
    assert getattr(c, call)() == D


def test_a_window_looks_back():
    c = Call()
    c.query.window, c.query.causal = 8, 0
    assert c.attend() == U


def test_workspace():
    c = Call(n=1, N=1)
    c.step.max_new, c.step.max_context, c.step.max_blocks = 1, 100000, 100000 // 16 + 1
    need = kvc.load().kvc_attend_workspace_bytes(c._ref("cache"), c._ref("step"), 8)
    assert need > 0  # one token and a long context: the ranges of it meet in the workspace
    for ws, size in ((None, need), (FAKE, 0), (FAKE, 255), (FAKE + 128, 1 << 30)):
        c.ws, c.ws_bytes = ws, size
        assert c.attend() == W
    lib = kvc.load()
    assert lib.kvc_attend_workspace_bytes(None, c._ref("step"), 8) == 0
    assert lib.kvc_attend_workspace_bytes(c._ref("cache"), None, 8) == 0
    for heads in (0, -2, 7):
        assert lib.kvc_attend_workspace_bytes(c._ref("cache"), c._ref("step"), heads) == 0
    c.step.max_context = -1
    assert lib.kvc_attend_workspace_bytes(c._ref("cache"), c._ref("step"), 8) == 0


@pytest.mark.parametrize("dtype", [kvc.KVC_F32, kvc.KVC_BF16, kvc.KVC_I8])
def test_nothing_to_do(dtype):
    """No rows, with or without sequences, is no error, and no layers is none for the moves; nothing is launched."""
    for n in (0, 2):
        c = Call(dtype=dtype)
        if dtype == kvc.KVC_F32:
            for f in ("block_stride", "token_stride", "head_stride"):
                assert getattr(c.cache, f) * 4 % 16 == 0
        c.step.num_seqs, c.step.num_rows, c.step.max_new = n, 0, 0
        c.rows.k = c.rows.v = c.query.q = c.query.out = None
        c.ws, c.ws_bytes = None, 0
        assert c.append() == c.gather() == c.attend() == kvc.KVC_OK
    c = Call(dtype=dtype)
    c.layers = (1, 1)
    assert c.append() == c.gather() == kvc.KVC_OK


def test_8_bit_caches_are_for_the_served_step():
    """The corrections read and write float32 and bfloat16 rows."""
    c = Call(dtype=kvc.KVC_I8)
    items = (kvc.kvc_item * 1)()
    items[0].num_tokens = 8
    items[0].state = kvc.kvc_state(2, 2, 128, 8, 16, kvc.KVC_BF16, kvc.KVC_GROUP_HEAD, 0, FAKE, FAKE, FAKE)
    batch = kvc.kvc_batch(1, 0, ctypes.cast(items, ctypes.POINTER(kvc.kvc_item)), FAKE, None, None)
    lib = kvc.load()
    assert lib.kvc_apply(c._ref("cache"), ctypes.byref(batch), 0, 2, None) == D
    assert lib.kvc_fit_state(c._ref("cache"), ctypes.byref(batch), 0, 2, kvc.KVC_FIT_DELTA, FAKE, 1 << 40,
                             None) == D


def host_cache(dtype=torch.bfloat16, **kw):
    pool = torch.zeros(4, 16, 2, 64, dtype=dtype)
    return kvc.Cache([pool], [pool], **kw)


def test_binding_cache_scales():
    pool = torch.zeros(4, 16, 2, 64, dtype=torch.int8)
    good = torch.zeros(4, 2, 16).permute(0, 2, 1)
    assert kvc.Cache([pool], [pool], k_scales=[good], v_scales=[good]).c.dtype == kvc.KVC_I8
    for k, v in (([good], None), (None, [good]), ([good], [good.double()]), ([good], [good.contiguous()]),
                 ([good[:, :8]], [good[:, :8]]), ([good, good], [good, good])):
        with pytest.raises(ValueError):
            kvc.Cache([pool], [pool], k_scales=k, v_scales=v)


def test_binding_step():
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)
    for bad in (lambda: kvc.Step([1, 1], [3], device="cpu"), lambda: kvc.Step([1], [3], offsets=[0, 1], device="cpu"),
                lambda: kvc.Step([1], [3], torch.zeros(2, 3, dtype=torch.int32)),
                lambda: kvc.Step([1], [3], torch.zeros(3, dtype=torch.int32)),
                lambda: kvc.Step.on_device(i32(0, 1), i32(3, 4), 1, 1, 3),
                lambda: kvc.Step.on_device(i32(0, 1).long(), i32(3), 1, 1, 3),
                lambda: kvc.Step.on_device(i32(0, 1), i32(3), 1, 1, 3, offsets=i32(1, 2)),
                lambda: kvc.Step.on_device(i32(0, 9, 1)[::2], i32(3), 1, 1, 3)):
        with pytest.raises(ValueError):
            bad()
    s = kvc.Step([2, 0, 3], [5, 0, 9], offsets=[0, 0, 4], device="cpu")
    assert s.num_rows == 5 and s.c.max_new == 3 and s.c.max_context == 9
    assert s.starts.tolist() == [0, 2, 2, 5] and s.contexts.tolist() == [5, 0, 9] and s.offsets.tolist() == [0, 0, 4]
    assert kvc.Step([], [], device="cpu").num_rows == 0
    assert kvc.Step([1], [1], offsets=[0], device="cpu").offsets is None


@pytest.mark.parametrize("shape_k,shape_v,dt_k,dt_v", [
    ((3, 2, 64), (3, 2, 64), torch.bfloat16, torch.float32), ((3, 2, 64), (3, 2, 64), torch.float16, torch.float16),
    ((4, 2, 64), (4, 2, 64), torch.bfloat16, torch.bfloat16), ((3, 2, 64), (4, 2, 64), torch.bfloat16, torch.bfloat16),
    ((3, 2, 32), (3, 2, 32), torch.bfloat16, torch.bfloat16), ((3, 1, 64), (3, 1, 64), torch.bfloat16, torch.bfloat16),
    ((2, 3, 2, 64), (2, 3, 2, 64), torch.bfloat16, torch.bfloat16), ((3, 128), (3, 128), torch.bfloat16, torch.bfloat16)])
def test_binding_rows(shape_k, shape_v, dt_k, dt_v):
    cache, step = host_cache(), kvc.Step([1, 2], [4, 5], device="cpu")
    k, v = torch.zeros(shape_k, dtype=dt_k), torch.zeros(shape_v, dtype=dt_v)
    for call in (kvc.kvc_append, kvc.kvc_gather):
        with pytest.raises(ValueError):
            call(cache, step, k, v)


def test_binding_refuses_host_memory_and_strided_elements():
    cache, step = host_cache(), kvc.Step([1, 2], [4, 5], device="cpu")
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    odd = torch.zeros(3, 2, 128, dtype=torch.bfloat16)[..., ::2]
    for call in (kvc.kvc_append, kvc.kvc_gather):
        with pytest.raises(ValueError, match="one GPU"):
            call(cache, step, k, k)
        with pytest.raises(ValueError, match="contiguous"):
            call(cache, step, odd, odd)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="one GPU"):
        kvc.kvc_attend(cache, step, q)
    for bad in (dict(q=q[:2]), dict(q=q[..., :32]), dict(q=q.half()), dict(q=q, out=q.float()), dict(q=q, out=q[:, :2]),
                dict(q=q, lse=torch.zeros(3, 4, dtype=torch.float64)), dict(q=q, lse=torch.zeros(4, 3).t()),
                dict(q=q, lse=torch.zeros(3, 2)), dict(q=q[0])):
        with pytest.raises(ValueError):
            kvc.kvc_attend(cache, step, **bad)


def test_workspace_of_a_cache_that_is_refused():
    c = Call(n=1, N=1)
    c.step.max_new, c.step.max_context, c.step.max_blocks = 1, 100000, 100000 // 16 + 1
    for d in (0, -128, 96, 1 << 30):
        c.cache.head_dim = d
        assert kvc.load().kvc_attend_workspace_bytes(c._ref("cache"), c._ref("step"), 8) == 0
