"""Python binding of libkvc (ctypes): argument marshalling only.

The names mirror the C ABI in include/kvc.h: kvc_fit_state, kvc_apply, kvc_chain, the anchor-pool calls
(kvc_anchor_weights, kvc_apply_anchored, kvc_gate_distances, kvc_gate_decide, kvc_pool_*), the served step
(kvc_append, kvc_gather, kvc_attend, kvc_rotate), a step of drafted tokens (kvc_tree, kvc_attend_tree, kvc_verify,
kvc_keep) and the size queries.  Every step
of the correction runs in the library's HIP kernels; torch only provides device memory and the stream.  Loading
fails loudly when the library has not been built.
"""
from __future__ import annotations

import collections
import ctypes
import functools
import math
import os
import struct
import threading
from typing import Deque, Dict, List, Optional, Sequence, Tuple

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libkvc.so")

KVC_OK, KVC_ERR_NULL_ARG, KVC_ERR_SHAPE, KVC_ERR_DTYPE, KVC_ERR_ALIGN = 0, 1, 2, 3, 4
KVC_ERR_ALIAS, KVC_ERR_WORKSPACE, KVC_ERR_UNSUPPORTED, KVC_ERR_HIP, KVC_ERR_TOO_LARGE = 5, 6, 7, 8, 9
KVC_NOALLOC_SCRATCH_BYTES = 2 << 20
KVC_F32, KVC_BF16, KVC_I8 = 0, 1, 2
KVC_FIT_DELTA, KVC_FIT_BASE = 0, 1
KVC_ROPE_NONE, KVC_ROPE_HALF, KVC_ROPE_PAIRS = 0, 1, 2
KVC_GROUP_HEAD, KVC_GROUP_LAYER = 0, 1
KVC_MAX_RANK = 128
KVC_MAX_ANCHORS = 16
KVC_MAX_TREE = 1024

EXPORTED = ["kvc_version", "kvc_status_str", "kvc_last_hip_error", "kvc_item_scratch_bytes", "kvc_state_bytes",
            "kvc_layer_state_bytes", "kvc_dense_bytes",
            "kvc_apply", "kvc_fit_workspace_bytes", "kvc_fit_state", "kvc_chain_workspace_bytes", "kvc_chain",
            "kvc_anchor_weights", "kvc_apply_anchored", "kvc_gate_workspace_bytes", "kvc_gate_distances",
            "kvc_gate_distances_noalloc",
            "kvc_gate_decide", "kvc_pool_create", "kvc_pool_destroy", "kvc_pool_insert", "kvc_pool_record_use",
            "kvc_pool_eligible", "kvc_pool_slot", "kvc_append", "kvc_gather", "kvc_attend_workspace_bytes",
            "kvc_attend_call_workspace_bytes", "kvc_attend", "kvc_rotate", "kvc_tree", "kvc_attend_tree", "kvc_verify_workspace_bytes", "kvc_verify",
            "kvc_keep"]


class KvcError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_str(status)} (status {status})")
        self.status = status


class kvc_cache(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("num_layers", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32), ("num_blocks", ctypes.c_int32),
                ("block_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("k_layers", ctypes.POINTER(ctypes.c_void_p)), ("v_layers", ctypes.POINTER(ctypes.c_void_p)),
                ("rope_style", ctypes.c_int32), ("rope_reserved", ctypes.c_int32),
                ("rope_inv_freq", ctypes.POINTER(ctypes.c_double))]


class kvc_state(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("num_tokens", ctypes.c_int32), ("rank", ctypes.c_int32), ("coef_dtype", ctypes.c_int),
                ("grouping", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("coef", ctypes.c_void_p), ("basis", ctypes.c_void_p), ("sigma", ctypes.c_void_p)]


class kvc_item(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int32), ("src_offset", ctypes.c_int32), ("dst_offset", ctypes.c_int32),
                ("src_position", ctypes.c_int32), ("dst_position", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("state", kvc_state)]


class kvc_batch(ctypes.Structure):
    _fields_ = [("num_items", ctypes.c_int32), ("max_blocks", ctypes.c_int32),
                ("items", ctypes.POINTER(kvc_item)), ("item_scratch", ctypes.c_void_p),
                ("src_tables", ctypes.c_void_p), ("dst_tables", ctypes.c_void_p)]


class kvc_anchors(ctypes.Structure):
    _fields_ = [("num_anchors", ctypes.c_int32), ("num_tokens", ctypes.c_int32),
                ("states", ctypes.POINTER(kvc_state)), ("weights", ctypes.c_void_p)]


class kvc_scales(ctypes.Structure):
    _fields_ = [("k_layers", ctypes.POINTER(ctypes.c_void_p)), ("v_layers", ctypes.POINTER(ctypes.c_void_p)),
                ("block_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class kvc_step(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("num_rows", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("max_context", ctypes.c_int32), ("max_blocks", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("starts", ctypes.c_void_p), ("contexts", ctypes.c_void_p), ("offsets", ctypes.c_void_p),
                ("tables", ctypes.c_void_p)]


class kvc_rows(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("reserved", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("layer_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class kvc_query(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("num_heads", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("window", ctypes.c_int32), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("q", ctypes.c_void_p), ("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("out", ctypes.c_void_p), ("out_token_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64),
                ("lse", ctypes.c_void_p)]


class kvc_heads(ctypes.Structure):
    _fields_ = [("num_heads", ctypes.c_int32), ("reserved", ctypes.c_int32), ("in_", ctypes.c_void_p),
                ("in_token_stride", ctypes.c_int64), ("in_head_stride", ctypes.c_int64), ("out", ctypes.c_void_p),
                ("out_token_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64)]


class kvc_rotary(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("num_rows", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("style", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("inverse", ctypes.c_int32),
                ("factor", ctypes.c_double), ("inv_freq", ctypes.c_void_p), ("positions", ctypes.c_void_p)]


class kvc_draft(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int32), ("children", ctypes.c_int32), ("parents", ctypes.c_void_p),
                ("tokens", ctypes.c_void_p), ("target", ctypes.c_void_p), ("target_stride", ctypes.c_int64),
                ("draft", ctypes.c_void_p), ("draft_stride", ctypes.c_int64), ("uniforms", ctypes.c_void_p),
                ("last", ctypes.c_void_p), ("path", ctypes.c_void_p), ("counts", ctypes.c_void_p),
                ("chosen", ctypes.c_void_p)]


_pack_rows = struct.Struct("@iiPPqqq").pack
_pack_query = struct.Struct("@iiiifiPqqPqqP").pack
_pack_heads = struct.Struct("@iiPqqPqq").pack
_pack_rotary = struct.Struct("@iiiiiidPP").pack
_pack_draft = struct.Struct("@iiPPPqPqPPPPP").pack
assert struct.calcsize("@iiPqqPqq") == ctypes.sizeof(kvc_heads)
assert struct.calcsize("@iiiiiidPP") == ctypes.sizeof(kvc_rotary)
assert struct.calcsize("@iiPPPqPqPPPPP") == ctypes.sizeof(kvc_draft)
assert struct.calcsize("@iiPPqqq") == ctypes.sizeof(kvc_rows)
assert struct.calcsize("@iiiifiPqqPqqP") == ctypes.sizeof(kvc_query)

_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libkvc.so (built by build.py).  Raises if it is missing: there is no fallback path."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2609_34060_amd/build.py (hipcc, gfx950)")
    lib = ctypes.CDLL(path)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    lib.kvc_version.restype = i32
    lib.kvc_status_str.restype = ctypes.c_char_p
    lib.kvc_status_str.argtypes = [ctypes.c_int]
    lib.kvc_last_hip_error.restype = i32
    lib.kvc_item_scratch_bytes.restype = sz
    lib.kvc_item_scratch_bytes.argtypes = [i32]
    lib.kvc_state_bytes.restype = sz
    lib.kvc_state_bytes.argtypes = [i32, i32, i32, i32, i32, ctypes.c_int]
    lib.kvc_layer_state_bytes.restype = sz
    lib.kvc_layer_state_bytes.argtypes = [i32, i32, i32, i32, i32, ctypes.c_int]
    lib.kvc_dense_bytes.restype = sz
    lib.kvc_dense_bytes.argtypes = [i32, i32, i32, i32, ctypes.c_int]
    lib.kvc_apply.restype = ctypes.c_int
    lib.kvc_apply.argtypes = [ctypes.POINTER(kvc_cache), ctypes.POINTER(kvc_batch), i32, i32, vp]
    lib.kvc_fit_workspace_bytes.restype = sz
    lib.kvc_fit_workspace_bytes.argtypes = [ctypes.POINTER(kvc_cache), ctypes.POINTER(kvc_batch), i32, i32]
    lib.kvc_fit_state.restype = ctypes.c_int
    lib.kvc_fit_state.argtypes = [ctypes.POINTER(kvc_cache), ctypes.POINTER(kvc_batch), i32, i32, ctypes.c_int,
                                  vp, sz, vp]
    lib.kvc_chain_workspace_bytes.restype = sz
    lib.kvc_chain_workspace_bytes.argtypes = [ctypes.POINTER(kvc_state)] * 3 + [i32, i32]
    lib.kvc_chain.restype = ctypes.c_int
    lib.kvc_chain.argtypes = [ctypes.POINTER(kvc_state)] * 3 + [i32, i32, vp, sz, vp]
    pc, pb, pa = ctypes.POINTER(kvc_cache), ctypes.POINTER(kvc_batch), ctypes.POINTER(kvc_anchors)
    f32, i64 = ctypes.c_float, ctypes.c_int64
    lib.kvc_anchor_weights.restype = ctypes.c_int
    lib.kvc_anchor_weights.argtypes = [pc, pb, pa, i32, i32, f32, vp]
    lib.kvc_apply_anchored.restype = ctypes.c_int
    lib.kvc_apply_anchored.argtypes = [pc, pb, pa, i32, i32, vp]
    lib.kvc_gate_workspace_bytes.restype = sz
    lib.kvc_gate_workspace_bytes.argtypes = [pc, pa, i32, i32, i32]
    lib.kvc_gate_distances.restype = ctypes.c_int
    lib.kvc_gate_distances.argtypes = [pc, pb, pa, i32, i32, i32, vp, vp, sz, vp]
    lib.kvc_gate_distances_noalloc.restype = ctypes.c_int
    lib.kvc_gate_distances_noalloc.argtypes = [pc, pb, pa, i32, i32, i32, vp, vp]
    lib.kvc_gate_decide.restype = i32
    lib.kvc_gate_decide.argtypes = [ctypes.POINTER(f32), i32, f32, f32, ctypes.POINTER(f32), ctypes.POINTER(f32)]
    lib.kvc_pool_create.restype = vp
    lib.kvc_pool_create.argtypes = [i32]
    lib.kvc_pool_destroy.restype = None
    lib.kvc_pool_destroy.argtypes = [vp]
    lib.kvc_pool_insert.restype = i32
    lib.kvc_pool_insert.argtypes = [vp, i64, i32, ctypes.POINTER(i64)]
    lib.kvc_pool_record_use.restype = ctypes.c_int
    lib.kvc_pool_record_use.argtypes = [vp, ctypes.POINTER(i32), i32]
    lib.kvc_pool_eligible.restype = i32
    lib.kvc_pool_eligible.argtypes = [vp, i32, ctypes.POINTER(i32)]
    lib.kvc_pool_slot.restype = ctypes.c_int
    lib.kvc_pool_slot.argtypes = [vp, i32, ctypes.POINTER(i64), ctypes.POINTER(i32), ctypes.POINTER(i64)]
    # the served step's calls are made for every layer of every step: addresses as plain integers, structs as bytes
    lib.kvc_append.restype = ctypes.c_int
    lib.kvc_append.argtypes = [vp, vp, vp, ctypes.c_char_p, i32, i32, vp]
    lib.kvc_gather.restype = ctypes.c_int
    lib.kvc_gather.argtypes = [vp, vp, vp, ctypes.c_char_p, i32, i32, vp]
    lib.kvc_attend_workspace_bytes.restype = sz
    lib.kvc_attend_workspace_bytes.argtypes = [vp, vp, i32]
    lib.kvc_attend_call_workspace_bytes.restype = sz
    lib.kvc_attend_call_workspace_bytes.argtypes = [vp, vp, i32, i32]
    lib.kvc_attend.restype = ctypes.c_int
    lib.kvc_attend.argtypes = [vp, vp, vp, ctypes.c_char_p, i32, vp, sz, vp]
    lib.kvc_rotate.restype = ctypes.c_int
    lib.kvc_rotate.argtypes = [ctypes.c_char_p, ctypes.c_char_p, ctypes.c_char_p, vp]
    lib.kvc_tree.restype = ctypes.c_int
    lib.kvc_tree.argtypes = [vp, vp, vp, i32, vp, vp]
    lib.kvc_attend_tree.restype = ctypes.c_int
    lib.kvc_attend_tree.argtypes = [vp, vp, vp, ctypes.c_char_p, vp, i32, i32, vp, sz, vp]
    lib.kvc_verify_workspace_bytes.restype = sz
    lib.kvc_verify_workspace_bytes.argtypes = [vp, i32]
    lib.kvc_verify.restype = ctypes.c_int
    lib.kvc_verify.argtypes = [vp, ctypes.c_char_p, vp, sz, vp]
    lib.kvc_keep.restype = ctypes.c_int
    lib.kvc_keep.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp]
    _lib = lib
    return lib


def status_str(status: int) -> str:
    return load().kvc_status_str(status).decode()


def _check(status: int, what: str) -> None:
    if status != KVC_OK:
        raise KvcError(status, what)


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.bfloat16:
        return KVC_BF16
    if dt == torch.float32:
        return KVC_F32
    raise ValueError(f"unsupported dtype {dt}")


def _stream_handle(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


# The library copies the host items (pinned memory) of a batch of several into its device scratch on the call's stream,
# so the copy reads the host bytes only when the stream reaches it, and the kernels read the batch's tables and states.
# A Batch passed as a temporary would be freed on return and its pinned block handed to the next allocation before that;
# calls that use a batch's items therefore keep it alive until an event recorded after the call has completed.  A
# stream's events complete in order, so each call looks at the oldest ones only (of every stream), and a completed event
# serves again: a call that queried every event in flight and made a new one spent more host time the more were queued.
_inflight: Dict[Tuple[int, int], Deque] = {}
_inflight_lock = threading.Lock()


def _hold_until_done(stream, batch: "Batch") -> None:
    if batch._host is None:
        return
    st = torch.cuda.current_stream() if stream is None else stream
    key = (st.device_index, st.cuda_stream)
    with _inflight_lock:
        free = None
        for k in list(_inflight):
            held = _inflight[k]
            while held and held[0][0].query():
                done = held.popleft()[0]
                if k == key:
                    free = done
            if not held and k != key:
                del _inflight[k]
        ev = torch.cuda.Event() if free is None else free
        ev.record(st)
        _inflight.setdefault(key, collections.deque()).append((ev, batch))


# ------------------------------------------------------------------------------------------------------------------
# Python-side holders (keep the tensors and ctypes arrays alive for the duration of a call)
# ------------------------------------------------------------------------------------------------------------------

class Cache:
    """kvc_cache over per-layer pools [num_blocks, block_size, num_kv_heads, head_dim] (or any strided view whose
    head_dim is contiguous).  rope_style / rope_inv_freq describe a rotary encoding of the key rows
    (KVC_ROPE_NONE: none).  int8 pools make an 8-bit cache (kvc_append, kvc_gather and kvc_attend take it), with the
    rows' float32 scales per layer in k_scales / v_scales, [num_blocks, block_size, num_kv_heads] or any strided view of
    that shape (attention reads a head's scales token after token: [num_blocks, num_kv_heads, block_size] in memory)."""

    def __init__(self, k_pools: Sequence[torch.Tensor], v_pools: Sequence[torch.Tensor],
                 strides: Optional[Sequence[int]] = None, rope_style: int = 0,
                 rope_inv_freq: Optional[Sequence[float]] = None,
                 k_scales: Optional[Sequence[torch.Tensor]] = None, v_scales: Optional[Sequence[torch.Tensor]] = None):
        assert len(k_pools) == len(v_pools) and len(k_pools) > 0
        p0 = k_pools[0]
        self.k_pools, self.v_pools = list(k_pools), list(v_pools)
        nb, bs, H, d = p0.shape
        if strides is None:
            strides = (p0.stride(0), p0.stride(1), p0.stride(2))
        n = len(k_pools)
        self._k = (ctypes.c_void_p * n)(*[p.data_ptr() for p in k_pools])
        self._v = (ctypes.c_void_p * n)(*[p.data_ptr() for p in v_pools])
        self._inv_freq = None
        if rope_inv_freq is not None:
            self._inv_freq = (ctypes.c_double * len(rope_inv_freq))(*[float(x) for x in rope_inv_freq])
        dtype = KVC_I8 if p0.dtype == torch.int8 else _dtype_code(p0.dtype)
        self.scales, self._scales_at = None, None
        if k_scales is not None or v_scales is not None:
            self._set_scales(k_scales, v_scales, (nb, bs, H))
        self.c = kvc_cache(dtype, n, H, d, bs, nb, strides[0], strides[1], strides[2],
                           ctypes.cast(self._k, ctypes.POINTER(ctypes.c_void_p)),
                           ctypes.cast(self._v, ctypes.POINTER(ctypes.c_void_p)), int(rope_style), 0,
                           None if self._inv_freq is None
                           else ctypes.cast(self._inv_freq, ctypes.POINTER(ctypes.c_double)))
        self._at = ctypes.addressof(self.c)
        self._layers, self._heads, self._dim = n, H, d
        # the GPU that holds all of it (-1: there is none)
        devices = {t.get_device() for t in self.k_pools + self.v_pools + (self.k_scales + self.v_scales if self.scales else [])}
        self._device = devices.pop() if len(devices) == 1 else -1

    def _set_scales(self, k_scales, v_scales, shape) -> None:
        if k_scales is None or v_scales is None:
            raise ValueError("k_scales and v_scales go together")
        s0 = k_scales[0]
        for s in [*k_scales, *v_scales]:
            if s.dtype != torch.float32 or tuple(s.shape) != tuple(shape) or s.stride() != s0.stride():
                raise ValueError("scales are float32 [num_blocks, block_size, num_kv_heads] of one layout")
        n = len(self.k_pools)
        if len(k_scales) != n or len(v_scales) != n:
            raise ValueError("one scale tensor for each layer's pool")
        self.k_scales, self.v_scales = list(k_scales), list(v_scales)
        self._ks = (ctypes.c_void_p * n)(*[s.data_ptr() for s in k_scales])
        self._vs = (ctypes.c_void_p * n)(*[s.data_ptr() for s in v_scales])
        self.scales = kvc_scales(ctypes.cast(self._ks, ctypes.POINTER(ctypes.c_void_p)),
                                 ctypes.cast(self._vs, ctypes.POINTER(ctypes.c_void_p)), *s0.stride())
        self._scales_at = ctypes.addressof(self.scales)

    @property
    def num_layers(self):
        return self.c.num_layers


class State:
    """Low-rank state tensors.  Per KV head: coef [L, 2, H, T, r], basis [L, 2, H, r, d] float32, sigma [L, 2, H, r].
    Per layer (KVC_GROUP_LAYER, recognised by a 4-d coef): coef [L, 2, T, r], basis [L, 2, r, H, d] float32 (a row
    of H d features), sigma [L, 2, r]."""

    def __init__(self, coef: torch.Tensor, basis: torch.Tensor, sigma: Optional[torch.Tensor] = None):
        self.coef, self.basis, self.sigma = coef, basis, sigma
        if coef.dim() == 4:
            L, two, T, r = coef.shape
            assert two == 2 and basis.dim() == 5 and basis.shape[:3] == (L, 2, r)
            H, d, grouping = basis.shape[3], basis.shape[4], KVC_GROUP_LAYER
        else:
            L, two, H, T, r = coef.shape
            assert two == 2 and basis.shape[:4] == (L, 2, H, r)
            d, grouping = basis.shape[-1], KVC_GROUP_HEAD
        self.grouping = grouping
        self.s = kvc_state(L, H, d, T, r, _dtype_code(coef.dtype), grouping, 0,
                           coef.data_ptr() if coef.numel() else None,
                           basis.data_ptr() if basis.numel() else None,
                           sigma.data_ptr() if (sigma is not None and sigma.numel()) else None)

    @staticmethod
    def empty(L: int, H: int, d: int, T: int, rank: int, coef_dtype: torch.dtype, device) -> "State":
        return State(torch.zeros(L, 2, H, T, rank, dtype=coef_dtype, device=device),
                     torch.zeros(L, 2, H, rank, d, dtype=torch.float32, device=device),
                     torch.zeros(L, 2, H, rank, dtype=torch.float32, device=device))

    @staticmethod
    def empty_layer(L: int, H: int, d: int, T: int, rank: int, coef_dtype: torch.dtype, device) -> "State":
        """A per-layer state (one factorisation of each layer's K or V rows, D = H d)."""
        return State(torch.zeros(L, 2, T, rank, dtype=coef_dtype, device=device),
                     torch.zeros(L, 2, rank, H, d, dtype=torch.float32, device=device),
                     torch.zeros(L, 2, rank, dtype=torch.float32, device=device))

    @property
    def num_tokens(self) -> int:
        return self.s.num_tokens

    @property
    def rank(self) -> int:
        return self.s.rank


class Batch:
    """kvc_batch: host items, the device scratch the library copies them into, and the block tables (device int32
    [n, max_blocks] or None).  The host items sit in pinned memory when a GPU is present, so the library's copy runs
    asynchronously on the call's stream; a Batch is not modified after construction."""

    def __init__(self, num_tokens: Sequence[int], src_offsets: Sequence[int], dst_offsets: Sequence[int],
                 states: Sequence[State], src_tables: Optional[torch.Tensor] = None,
                 dst_tables: Optional[torch.Tensor] = None, device=None,
                 src_positions: Optional[Sequence[int]] = None, dst_positions: Optional[Sequence[int]] = None):
        n = len(num_tokens)
        self.states = list(states)
        nbytes = ctypes.sizeof(kvc_item) * max(n, 1)
        self._host = None
        if torch.cuda.is_available():
            self._host = torch.zeros(nbytes, dtype=torch.uint8, pin_memory=True)
            arr = (kvc_item * max(n, 1)).from_address(self._host.data_ptr())
        else:
            arr = (kvc_item * max(n, 1))()
        for i in range(n):
            arr[i].num_tokens = int(num_tokens[i])
            arr[i].src_offset = int(src_offsets[i])
            arr[i].dst_offset = int(dst_offsets[i])
            arr[i].src_position = 0 if src_positions is None else int(src_positions[i])
            arr[i].dst_position = 0 if dst_positions is None else int(dst_positions[i])
            arr[i].reserved = 0
            arr[i].state = states[i].s
        self._items = arr
        device = device if device is not None else (states[0].basis.device if n else "cuda")
        self.item_scratch = torch.empty(kvc_item_scratch_bytes(n), dtype=torch.uint8, device=device) if n else None
        self.src_tables = None if src_tables is None else src_tables.to(torch.int32).contiguous()
        self.dst_tables = None if dst_tables is None else dst_tables.to(torch.int32).contiguous()
        max_blocks = 0
        for t in (self.src_tables, self.dst_tables):
            if t is not None:
                assert t.shape[0] == n
                max_blocks = max(max_blocks, t.shape[1])
        if self.src_tables is not None and self.dst_tables is not None:
            assert self.src_tables.shape[1] == self.dst_tables.shape[1]
        self.b = kvc_batch(n, max_blocks, ctypes.cast(arr, ctypes.POINTER(kvc_item)),
                           self.item_scratch.data_ptr() if n else None,
                           None if self.src_tables is None else self.src_tables.data_ptr(),
                           None if self.dst_tables is None else self.dst_tables.data_ptr())


# ------------------------------------------------------------------------------------------------------------------
# Entry points (same names as the C ABI)
# ------------------------------------------------------------------------------------------------------------------

def kvc_version() -> int:
    return load().kvc_version()


def kvc_item_scratch_bytes(num_items: int) -> int:
    return load().kvc_item_scratch_bytes(num_items)


def kvc_state_bytes(L: int, H: int, d: int, T: int, rank: int, coef_dtype: int) -> int:
    return load().kvc_state_bytes(L, H, d, T, rank, coef_dtype)


def kvc_layer_state_bytes(L: int, H: int, d: int, T: int, rank: int, coef_dtype: int) -> int:
    return load().kvc_layer_state_bytes(L, H, d, T, rank, coef_dtype)


def kvc_dense_bytes(L: int, H: int, d: int, T: int, dtype: int) -> int:
    return load().kvc_dense_bytes(L, H, d, T, dtype)


def kvc_apply(cache: Cache, batch: Batch, layer_begin: int = 0, layer_end: Optional[int] = None,
              stream=None) -> None:
    layer_end = cache.num_layers if layer_end is None else layer_end
    stream = torch.cuda.current_stream() if stream is None else stream
    st = load().kvc_apply(ctypes.byref(cache.c), ctypes.byref(batch.b), layer_begin, layer_end,
                          _stream_handle(stream))
    _check(st, "kvc_apply")
    _hold_until_done(stream, batch)


def kvc_fit_workspace_bytes(cache: Cache, batch: Batch, layer_begin: int = 0, layer_end: Optional[int] = None) -> int:
    layer_end = cache.num_layers if layer_end is None else layer_end
    return load().kvc_fit_workspace_bytes(ctypes.byref(cache.c), ctypes.byref(batch.b), layer_begin, layer_end)


def kvc_fit_state(cache: Cache, batch: Batch, layer_begin: int = 0, layer_end: Optional[int] = None,
                  mode: int = KVC_FIT_DELTA, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    layer_end = cache.num_layers if layer_end is None else layer_end
    stream = torch.cuda.current_stream() if stream is None else stream
    if workspace is None:  # the call itself checks the size of a given one
        need = kvc_fit_workspace_bytes(cache, batch, layer_begin, layer_end)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=cache.k_pools[0].device)
    st = load().kvc_fit_state(ctypes.byref(cache.c), ctypes.byref(batch.b), layer_begin, layer_end, mode,
                              ctypes.c_void_p(workspace.data_ptr()), workspace.numel(), _stream_handle(stream))
    _check(st, "kvc_fit_state")
    _hold_until_done(stream, batch)


def kvc_chain_workspace_bytes(first: State, second: State, out: State, layer_begin: int = 0,
                              layer_end: Optional[int] = None) -> int:
    layer_end = first.s.num_layers if layer_end is None else layer_end
    return load().kvc_chain_workspace_bytes(ctypes.byref(first.s), ctypes.byref(second.s), ctypes.byref(out.s),
                                            layer_begin, layer_end)


def kvc_chain(first: State, second: State, out: State, layer_begin: int = 0, layer_end: Optional[int] = None,
              workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    layer_end = first.s.num_layers if layer_end is None else layer_end
    if workspace is None:
        need = kvc_chain_workspace_bytes(first, second, out, layer_begin, layer_end)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=first.basis.device)
    st = load().kvc_chain(ctypes.byref(first.s), ctypes.byref(second.s), ctypes.byref(out.s), layer_begin,
                          layer_end, ctypes.c_void_p(workspace.data_ptr()), workspace.numel(),
                          _stream_handle(stream))
    _check(st, "kvc_chain")


# ------------------------------------------------------------------------------------------------------------------
# Anchor pool (Section 3.3, Appendix A.3)
# ------------------------------------------------------------------------------------------------------------------

class Anchors:
    """kvc_anchors: the anchors' states (bases or delta corrections) and the weights tensor
    [layers, 2, num_tokens, V] float32 (allocated here when not given)."""

    def __init__(self, states: Sequence[State], num_tokens: int, num_layers: int,
                 weights: Optional[torch.Tensor] = None):
        self.states = list(states)
        V = len(self.states)
        self._arr = (kvc_state * max(V, 1))(*[st.s for st in self.states])
        if weights is None and V:
            weights = torch.empty(num_layers, 2, num_tokens, V, dtype=torch.float32,
                                  device=self.states[0].basis.device)
        self.weights = weights
        self.a = kvc_anchors(V, num_tokens, ctypes.cast(self._arr, ctypes.POINTER(kvc_state)),
                             None if weights is None or weights.numel() == 0 else weights.data_ptr())

    def with_states(self, states: Sequence[State]) -> "Anchors":
        """The same weights with other states (the delta corrections after the weights came from the bases)."""
        return Anchors(states, self.a.num_tokens, 0 if self.weights is None else self.weights.shape[0], self.weights)


def kvc_anchor_weights(cache: Cache, batch: Batch, anchors: Anchors, layer_begin: int = 0,
                       layer_end: Optional[int] = None, temperature: float = 1.0, stream=None) -> None:
    layer_end = cache.num_layers if layer_end is None else layer_end
    st = load().kvc_anchor_weights(ctypes.byref(cache.c), ctypes.byref(batch.b), ctypes.byref(anchors.a), layer_begin,
                                   layer_end, float(temperature), _stream_handle(stream))
    _check(st, "kvc_anchor_weights")


def kvc_apply_anchored(cache: Cache, batch: Batch, anchors: Anchors, layer_begin: int = 0,
                       layer_end: Optional[int] = None, stream=None) -> None:
    layer_end = cache.num_layers if layer_end is None else layer_end
    st = load().kvc_apply_anchored(ctypes.byref(cache.c), ctypes.byref(batch.b), ctypes.byref(anchors.a),
                                   layer_begin, layer_end, _stream_handle(stream))
    _check(st, "kvc_apply_anchored")


def kvc_gate_workspace_bytes(cache: Cache, anchors: Anchors, prefix: int, layer_begin: int = 0,
                             layer_end: Optional[int] = None) -> int:
    layer_end = cache.num_layers if layer_end is None else layer_end
    return load().kvc_gate_workspace_bytes(ctypes.byref(cache.c), ctypes.byref(anchors.a), prefix, layer_begin,
                                           layer_end)


def kvc_gate_distances(cache: Cache, batch: Batch, anchors: Anchors, prefix: int, layer_begin: int = 0,
                       layer_end: Optional[int] = None, distances: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    layer_end = cache.num_layers if layer_end is None else layer_end
    dev = cache.k_pools[0].device
    if distances is None:
        distances = torch.empty(len(anchors.states), dtype=torch.float32, device=dev)
    if workspace is None:
        need = kvc_gate_workspace_bytes(cache, anchors, prefix, layer_begin, layer_end)
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = load().kvc_gate_distances(ctypes.byref(cache.c), ctypes.byref(batch.b), ctypes.byref(anchors.a), prefix,
                                   layer_begin, layer_end, ctypes.c_void_p(distances.data_ptr()),
                                   ctypes.c_void_p(workspace.data_ptr()), workspace.numel(), _stream_handle(stream))
    _check(st, "kvc_gate_distances")
    return distances


def kvc_gate_distances_noalloc(cache: Cache, batch: Batch, anchors: Anchors, prefix: int, layer_begin: int = 0,
                               layer_end: Optional[int] = None, distances: Optional[torch.Tensor] = None,
                               stream=None) -> torch.Tensor:
    """kvc_gate_distances with the library's static scratch instead of a workspace: `distances` (float32 [V], on the
    device) must be passed by a caller that cannot allocate; it is allocated here only when omitted."""
    layer_end = cache.num_layers if layer_end is None else layer_end
    if distances is None:
        distances = torch.empty(len(anchors.states), dtype=torch.float32, device=cache.k_pools[0].device)
    st = load().kvc_gate_distances_noalloc(ctypes.byref(cache.c), ctypes.byref(batch.b), ctypes.byref(anchors.a),
                                           prefix, layer_begin, layer_end, ctypes.c_void_p(distances.data_ptr()),
                                           _stream_handle(stream))
    _check(st, "kvc_gate_distances_noalloc")
    return distances


def kvc_gate_decide(distances: Sequence[float], tau: float, temperature: float = 1.0):
    """Returns (accept, gate weights, normalised entropy) of Eq. 10-11 for host distances."""
    n = len(distances)
    d = (ctypes.c_float * max(n, 1))(*[float(x) for x in distances])
    g = (ctypes.c_float * max(n, 1))()
    h = ctypes.c_float()
    acc = load().kvc_gate_decide(d, n, float(tau), float(temperature), g, ctypes.byref(h))
    return bool(acc), [g[i] for i in range(n)], h.value


class Pool:
    """kvc_pool_*: the anchor bookkeeping of one shared-context slot (host only)."""

    def __init__(self, capacity: int):
        self.p = load().kvc_pool_create(capacity)
        if not self.p:
            raise KvcError(KVC_ERR_SHAPE, "kvc_pool_create")
        self.capacity = capacity

    def __del__(self):
        if getattr(self, "p", None) and _lib is not None:
            _lib.kvc_pool_destroy(self.p)
            self.p = None

    def insert(self, anchor_id: int, length: int):
        ev = ctypes.c_int64()
        slot = load().kvc_pool_insert(self.p, anchor_id, length, ctypes.byref(ev))
        if slot < 0:
            raise KvcError(KVC_ERR_SHAPE, "kvc_pool_insert")
        return slot, (None if ev.value < 0 else ev.value)

    def record_use(self, slots: Sequence[int]) -> None:
        arr = (ctypes.c_int32 * max(len(slots), 1))(*slots)
        _check(load().kvc_pool_record_use(self.p, arr, len(slots)), "kvc_pool_record_use")

    def eligible(self, prefix: int) -> List[int]:
        arr = (ctypes.c_int32 * self.capacity)()
        n = load().kvc_pool_eligible(self.p, prefix, arr)
        return [arr[i] for i in range(n)]

    def slot(self, slot: int):
        aid, length, uses = ctypes.c_int64(), ctypes.c_int32(), ctypes.c_int64()
        _check(load().kvc_pool_slot(self.p, slot, ctypes.byref(aid), ctypes.byref(length), ctypes.byref(uses)),
               "kvc_pool_slot")
        return aid.value, length.value, uses.value


# ------------------------------------------------------------------------------------------------------------------
# A served step: new tokens written into the cache, read back, attended with
# ------------------------------------------------------------------------------------------------------------------

class Step:
    """kvc_step: the new tokens of one step, the same for every layer of a model.  new_tokens[i] of them belong to
    sequence i (in this order in the calls' token-major arrays) and are the last of its contexts[i] tokens in the cache;
    its token t sits at position offsets[i] + t of the blocks tables[i] (device int32 [n, max_blocks]; None: the pool in
    order).  The lengths are copied to the device here, and so are tables of another type or layout."""

    def __init__(self, new_tokens: Sequence[int], contexts: Sequence[int], tables: Optional[torch.Tensor] = None,
                 offsets: Optional[Sequence[int]] = None, device=None):
        n = len(new_tokens)
        if len(contexts) != n or (offsets is not None and len(offsets) != n):
            raise ValueError("one context (and offset) for each sequence")
        device = device if device is not None else (tables.device if tables is not None else "cuda")
        host, at = [0], 0
        for q in new_tokens:
            at += int(q)
            host.append(at)
        host += [int(c) for c in contexts]
        offsets = None if offsets is None or not any(offsets) else offsets
        host += [] if offsets is None else [int(o) for o in offsets]
        # (the copy of the lengths waits for the current stream, and with it for that of the tables before it: calls on any
        # other stream find both whole)
        tables = None if tables is None else tables.to(torch.int32).contiguous()
        dev = torch.tensor(host, dtype=torch.int32, device=device)
        self._set(dev[:n + 1], dev[n + 1:2 * n + 1], at, max([int(q) for q in new_tokens], default=0),
                  max([int(c) for c in contexts], default=0), tables, None if offsets is None else dev[2 * n + 1:])

    @classmethod
    def on_device(cls, starts: torch.Tensor, contexts: torch.Tensor, num_rows: int, max_new: int, max_context: int,
                  tables: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None) -> "Step":
        """A step whose starts [n + 1], contexts [n], offsets [n] and tables [n, max_blocks] are on the device already
        (contiguous int32, taken as they are), under the host's bounds: a captured call then follows them from replay to
        replay."""
        self = cls.__new__(cls)
        self._set(starts, contexts, num_rows, max_new, max_context, tables, offsets)
        return self

    def _set(self, starts, contexts, num_rows, max_new, max_context, tables, offsets) -> None:
        n = contexts.numel()
        for t, size in ((starts, n + 1), (contexts, n), (offsets, n)):
            if t is not None and (t.dtype != torch.int32 or not t.is_contiguous() or t.numel() != size):
                raise ValueError("starts [n + 1], contexts [n] and offsets [n] are contiguous int32")
        if tables is not None:
            if tables.dim() != 2 or tables.shape[0] != n or tables.dtype != torch.int32 or not tables.is_contiguous():
                raise ValueError("tables is contiguous int32 [n, max_blocks]")
        self.starts, self.contexts, self.offsets, self.tables = starts, contexts, offsets, tables
        self.num_rows = int(num_rows)
        self.c = kvc_step(n, self.num_rows, int(max_new), int(max_context), 0 if tables is None else tables.shape[1], 0,
                          starts.data_ptr(), contexts.data_ptr(), None if offsets is None else offsets.data_ptr(),
                          None if tables is None else tables.data_ptr())
        self._at = ctypes.addressof(self.c)
        self._tensors = [t for t in (starts, contexts, offsets, tables) if t is not None]
        devices = {t.get_device() for t in self._tensors}
        self._device = devices.pop() if len(devices) == 1 else -1


@functools.lru_cache(maxsize=None)
def _several_gpus() -> bool:
    return torch.cuda.device_count() > 1


def _raw_stream(stream, cache: Cache, step: Step, a: torch.Tensor, b: torch.Tensor) -> int:
    """The given stream, or the current one of the device that holds everything.  A given stream may still read the
    step's arrays when the caller lets go of them."""
    dev = cache._device
    if dev < 0 or step._device != dev or a.get_device() != dev or b.get_device() != dev:
        raise ValueError("the cache, the step and the tensors of a call are on one GPU")
    return _stream_of(stream, dev, step._tensors)


def _stream_of(stream, dev: int, read: Sequence[torch.Tensor]) -> int:
    """The given stream of GPU dev, which may still read `read` when the caller lets go of it, or dev's current one."""
    # (kernels of a null stream run on the current GPU; to ask for it takes 0.4 us, which where there is one GPU is spared)
    if _several_gpus() and torch._C._cuda_getDevice() != dev:
        raise ValueError("a call's GPU is the current one")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        raise ValueError("the stream of a call is one of its GPU")
    for t in read:
        t.record_stream(stream)
    return stream.cuda_stream


def _tensors_stream(stream, step: Optional[Step], dev: int, tensors: Sequence[Optional[torch.Tensor]]) -> int:
    """_raw_stream for calls without a cache, whose tensors (those that are given) are on GPU dev."""
    for t in tensors:
        if t is not None and t.get_device() != dev:
            dev = -1
    if dev < 0:
        raise ValueError("the step and the tensors of a call are on one GPU")
    return _stream_of(stream, dev, () if step is None else step._tensors)


def _allocate(stream, make):
    """make() in memory of the call's own stream: what the current one still does with a block that it freed is not
    waited for."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        return make()


def _plain(t: torch.Tensor, dtype: torch.dtype, shape, what: str) -> int:
    """The address of a contiguous tensor of that type and shape."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} is contiguous {str(dtype)[6:]} {list(shape)}: got {t.dtype} {list(t.shape)}")
    return t.data_ptr()


_SERVE_DTYPE = {torch.float32: KVC_F32, torch.bfloat16: KVC_BF16}


def _move_rows(call, name: str, cache: Cache, step: Step, k: torch.Tensor, v: torch.Tensor, layer_begin: int,
               layer_end: Optional[int], stream) -> None:
    layer_end = cache._layers if layer_end is None else layer_end
    st, shape, torch_dtype = k.stride(), k.shape, k.dtype
    dtype = _SERVE_DTYPE.get(torch_dtype)
    if dtype is None or v.dtype != torch_dtype or v.shape != shape or v.stride() != st:
        raise ValueError("k and v are float32 or bfloat16 of one shape, layout and dtype")
    if len(st) == 3:
        st, shape = (0, *st), (1, *shape)
    layers, tokens, heads, dim = shape if len(st) == 4 else (0, -1, 0, 0)
    if layers != layer_end - layer_begin or tokens != step.num_rows or heads != cache._heads or dim != cache._dim:
        raise ValueError(f"rows are [layers, N, num_kv_heads, head_dim], [N, num_kv_heads, head_dim] for one layer: got "
                         f"{tuple(k.shape)} for {layer_end - layer_begin} layers, N = {step.num_rows}")
    if st[3] != 1 and k.numel():
        raise ValueError("head_dim is contiguous in k and v")
    status = call(cache._at, cache._scales_at, step._at,
                  _pack_rows(dtype, 0, k.data_ptr(), v.data_ptr(), st[0], st[1], st[2]), layer_begin, layer_end,
                  _raw_stream(stream, cache, step, k, v))
    if status:
        raise KvcError(status, name)


def kvc_append(cache: Cache, step: Step, k: torch.Tensor, v: torch.Tensor, layer_begin: int = 0,
               layer_end: Optional[int] = None, stream=None) -> None:
    """Writes the step's rows k, v [layers, N, num_kv_heads, head_dim] (any strides with head_dim contiguous) into the
    cache, quantised where the cache is int8."""
    _move_rows(load().kvc_append, "kvc_append", cache, step, k, v, layer_begin, layer_end, stream)


def kvc_gather(cache: Cache, step: Step, k: torch.Tensor, v: torch.Tensor, layer_begin: int = 0,
               layer_end: Optional[int] = None, stream=None) -> None:
    """Reads the step's tokens from the cache into k, v: the inverse of kvc_append."""
    _move_rows(load().kvc_gather, "kvc_gather", cache, step, k, v, layer_begin, layer_end, stream)


def kvc_attend_workspace_bytes(cache: Cache, step: Step, num_heads: int, tree: Optional[bool] = None) -> int:
    """The workspace that serves kvc_attend and kvc_attend_tree alike, or with `tree` False or True the one of them alone."""
    if tree is None:
        return load().kvc_attend_workspace_bytes(cache._at, step._at, num_heads)
    return load().kvc_attend_call_workspace_bytes(cache._at, step._at, num_heads, 1 if tree else 0)


def _attend_memory(lib, cache, step, q, heads, out, workspace, tree):
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if workspace is None:  # the call itself checks the size of a given one
        workspace = torch.empty(lib.kvc_attend_call_workspace_bytes(cache._at, step._at, heads, tree), dtype=torch.uint8,
                                device=q.device)
    return out, workspace


def kvc_attend(cache: Cache, step: Step, q: torch.Tensor, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None, layer: int = 0, scale: Optional[float] = None, causal: bool = True,
               window: int = 0, workspace: Optional[torch.Tensor] = None, stream=None, *,
               _masks: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the step's queries q [N, num_heads, head_dim] over one layer of the cache; returns out (allocated
    here when not given).  lse (float32 [N, num_heads]) receives the log-sum-exp of the scores where it is given.  Rows that
    belong to no sequence of the step are left as they are (undefined where out is allocated here)."""
    shape, torch_dtype, qs = q.shape, q.dtype, q.stride()
    N, heads, d = shape
    dtype = _SERVE_DTYPE.get(torch_dtype)
    if N != step.num_rows or d != cache._dim or dtype is None or (
            out is not None and (out.shape != shape or out.dtype != torch_dtype)):
        raise ValueError("q and out are float32 or bfloat16 [N, num_heads, head_dim]")
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != (N, heads) or not lse.is_contiguous()):
        raise ValueError("lse is contiguous float32 [N, num_heads]")
    lib = load()
    raw = _raw_stream(stream, cache, step, q, q if out is None else out)
    if lse is not None or workspace is not None:
        _raw_stream(stream, cache, step, q if lse is None else lse, q if workspace is None else workspace)
    tree = 0 if _masks is None else 1
    if stream is not None and (out is None or workspace is None):
        # (memory of the call's own stream: what the current one still does with a block that it freed is not waited for)
        with torch.cuda.stream(stream):
            out, workspace = _attend_memory(lib, cache, step, q, heads, out, workspace, tree)
    else:
        out, workspace = _attend_memory(lib, cache, step, q, heads, out, workspace, tree)
    os_ = out.stride()
    if (qs[2] != 1 or os_[2] != 1) and q.numel():
        raise ValueError("head_dim is contiguous in q and out")
    query = _pack_query(dtype, heads, 1 if causal else 0, window, d ** -0.5 if scale is None else scale, 0,
                        q.data_ptr(), qs[0], qs[1], out.data_ptr(), os_[0], os_[1],
                        0 if lse is None else lse.data_ptr())
    room = workspace.numel() * workspace.element_size()
    if _masks is None:
        status = lib.kvc_attend(cache._at, cache._scales_at, step._at, query, layer, workspace.data_ptr(), room, raw)
    else:
        status = lib.kvc_attend_tree(cache._at, cache._scales_at, step._at, query, _masks.data_ptr(), _masks.shape[1],
                                     layer, workspace.data_ptr(), room, raw)
    if status:
        raise KvcError(status, "kvc_attend" if _masks is None else "kvc_attend_tree")
    return out


# ------------------------------------------------------------------------------------------------------------------
# Rotary positions
# ------------------------------------------------------------------------------------------------------------------

def rope_frequencies(rotary_dim: int, theta: float = 10000.0, scale: float = 1.0, trained: Optional[int] = None,
                     slow: float = 1.0, fast: float = 32.0) -> List[float]:
    """theta^(-2 i / rotary_dim) for each feature pair, for contexts `scale` times as long as the trained ones.  With
    `trained` (the trained context) only pairs that make up to `slow` turns over it are slowed by all of scale, those of
    `fast` turns or more are kept, and a ramp of the turns lies between; without it every pair is slowed.  The rotated
    features are usually multiplied by rope_factor(scale) in the former case (Rotary's factor)."""
    if rotary_dim < 2 or rotary_dim % 2 or not theta > 0 or not scale > 0 or not fast > slow:
        raise ValueError("an even rotary_dim, positive theta and scale, and fast above slow")
    freq = [theta ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)]
    if trained is None:
        return [f / scale for f in freq]
    keep = [min(1.0, max(0.0, (trained * f / (2.0 * math.pi) - slow) / (fast - slow))) for f in freq]
    return [f * k + f / scale * (1.0 - k) for f, k in zip(freq, keep)]


def rope_factor(scale: float) -> float:
    """0.1 ln(scale) + 1, at least 1: by how much the rotated features grow in a context `scale` times the trained one."""
    return 0.1 * math.log(max(scale, 1.0)) + 1.0


class Rotary:
    """kvc_rotary without its rows: the frequencies of the feature pairs (radians per position), the head dimension, the
    layout of the pairs and the factor of the rotated features.  The first 2 * len(inv_freq) features are rotated."""

    def __init__(self, inv_freq: Sequence[float], head_dim: int, style: int = KVC_ROPE_HALF, factor: float = 1.0):
        self.head_dim, self.style, self.factor = int(head_dim), int(style), float(factor)
        self.rotary_dim = 2 * len(inv_freq)
        self._inv_freq = (ctypes.c_double * max(1, len(inv_freq)))(*[float(x) for x in inv_freq])
        self._at = ctypes.addressof(self._inv_freq)


def _pack_rotated(x: torch.Tensor, out: torch.Tensor, shape) -> bytes:
    n, heads, _ = shape
    (xn, xh, xd), (on, oh, od) = x.stride(), out.stride()
    if (xd != 1 or od != 1) and n and heads:
        raise ValueError("head_dim is contiguous in the rows and their results")
    if n <= 1:  # (the stride of one row is any)
        xn = on = 0
    if heads <= 1:
        xh = oh = 0
    return _pack_heads(heads, 0, x.data_ptr(), xn, xh, out.data_ptr(), on, oh)


def kvc_rotate(rotary: Rotary, positions: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, inverse: bool = False,
               stream=None):
    """The rows q [N, heads, head_dim] and, in the same launch, k (another number of heads) rotated to positions [N]
    (int32); with `inverse` to -positions, which takes gradients back.  Returns q_out, or (q_out, k_out) where k is given
    (allocated here when not given; they may be q and k themselves).  As every call here it is outside autograd: a result
    carries no graph, and the gradient of q is that of the result rotated with `inverse`."""
    shape, torch_dtype = q.shape, q.dtype
    dtype = _SERVE_DTYPE.get(torch_dtype)
    if dtype is None or len(shape) != 3 or shape[2] != rotary.head_dim or (
            q_out is not None and (q_out.shape != shape or q_out.dtype is not torch_dtype)):
        raise ValueError("q, k and their results are float32 or bfloat16 [N, heads, head_dim]")
    if k is None:
        if k_out is not None:
            raise ValueError("k_out goes with k")
    else:
        k_shape = k.shape
        if len(k_shape) != 3 or k_shape[0] != shape[0] or k_shape[2] != shape[2] or k.dtype is not torch_dtype or (
                k_out is not None and (k_out.shape != k_shape or k_out.dtype is not torch_dtype)):
            raise ValueError("q, k and their results are float32 or bfloat16 [N, heads, head_dim]")
    at = _plain(positions, torch.int32, shape[:1], "positions")
    raw = _tensors_stream(stream, None, q.get_device(), (positions, k, q_out, k_out))
    if q_out is None:
        q_out = _allocate(stream, lambda: torch.empty_like(q, memory_format=torch.contiguous_format))
    if k_out is None and k is not None:
        k_out = _allocate(stream, lambda: torch.empty_like(k, memory_format=torch.contiguous_format))
    status = load().kvc_rotate(
        _pack_rotary(dtype, shape[0], rotary.head_dim, rotary.style, rotary.rotary_dim, 1 if inverse else 0,
                     rotary.factor, rotary._at, at),
        _pack_rotated(q, q_out, shape), None if k is None else _pack_rotated(k, k_out, k_shape), raw)
    if status:
        raise KvcError(status, "kvc_rotate")
    return q_out if k is None else (q_out, k_out)


# ------------------------------------------------------------------------------------------------------------------
# A step of drafted tokens
# ------------------------------------------------------------------------------------------------------------------

def kvc_tree(step: Step, parents: torch.Tensor, masks: Optional[torch.Tensor] = None,
             positions: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Each new token's ancestors as bits, masks int64 [N, words] with 64 words >= step's max_new, and its position, int32
    [N], from parents int32 [N] (a token's parent among its sequence's new tokens; -1: none).  The results are allocated
    here when not given; rows of no sequence are left as they are (undefined where they are allocated here)."""
    N = step.num_rows
    at = _plain(parents, torch.int32, (N,), "parents")
    raw = _tensors_stream(stream, step, step._device, (parents, masks, positions))
    if masks is None:
        masks = _allocate(stream, lambda: torch.empty(N, max(1, (step.c.max_new + 63) // 64), dtype=torch.int64,
                                                      device=parents.device))
    if positions is None:
        positions = _allocate(stream, lambda: torch.empty(N, dtype=torch.int32, device=parents.device))
    if masks.dim() != 2:
        raise ValueError("masks is int64 [N, words]")
    status = load().kvc_tree(step._at, at, _plain(masks, torch.int64, (N, masks.shape[1]), "masks"), masks.shape[1],
                             _plain(positions, torch.int32, (N,), "positions"), raw)
    if status:
        raise KvcError(status, "kvc_tree")
    return masks, positions


def kvc_attend_tree(cache: Cache, step: Step, masks: torch.Tensor, q: torch.Tensor, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, layer: int = 0, scale: Optional[float] = None, window: int = 0,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """kvc_attend for drafted tokens: each sees the context before the step's new tokens, and of these the ones that its
    mask (int64 [N, words], kvc_tree's) names.  The workspace is of kvc_attend_workspace_bytes."""
    if masks.dim() != 2:
        raise ValueError("masks is int64 [N, words]")
    _plain(masks, torch.int64, (step.num_rows, masks.shape[1]), "masks")
    if masks.get_device() != cache._device:
        raise ValueError("the cache, the step and the tensors of a call are on one GPU")
    return kvc_attend(cache, step, q, out, lse, layer, scale, True, window, workspace, stream, _masks=masks)


def kvc_verify_workspace_bytes(step: Step, vocab: int) -> int:
    return load().kvc_verify_workspace_bytes(step._at, vocab)


def _pack_probabilities(x: Optional[torch.Tensor], N: int, vocab: int, what: str) -> Tuple[int, int]:
    if x is None:
        return 0, 0
    if x.dtype is not torch.float32 or x.shape != (N, vocab):
        raise ValueError(f"{what} is float32 [N, vocab]")
    row, one = x.stride()
    if one != 1 and vocab > 1 and N:
        raise ValueError(f"the probabilities of a row of {what} are next to one another")
    return x.data_ptr(), max(vocab, row) if N <= 1 else row


def kvc_verify(step: Step, parents: torch.Tensor, tokens: torch.Tensor, target: torch.Tensor, uniforms: torch.Tensor,
               last: torch.Tensor, draft: Optional[torch.Tensor] = None, children: int = 0,
               path: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
               chosen: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
               stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Which drafted tokens the target accepts.  parents and tokens are int32 [N] (token 0 of a sequence is the one that is
    settled already), target float32 [N, vocab] holds the target's probabilities after each token and draft those that a
    token's children were drawn from (None: they were not drawn); uniforms float32 [N] and last float32 [num_seqs] are
    random numbers.  At most `children` children of a token are tried (0: all); one is the quicker for drawn tokens.
    Returns path [N] (a sequence's accepted tokens in its first rows, then -1), counts [num_seqs] and chosen [num_seqs], the
    token after the accepted ones (int32, allocated here when not given)."""
    N, n, vocab = step.num_rows, step.contexts.numel(), target.shape[-1]
    raw = _tensors_stream(stream, step, step._device,
                          (parents, tokens, target, uniforms, last, draft, path, counts, chosen, workspace))
    lib = load()

    if path is None or counts is None or chosen is None or workspace is None:
        def missing():
            new = [torch.empty(size, dtype=torch.int32, device=parents.device) if t is None else t
                   for t, size in ((path, N), (counts, n), (chosen, n))]
            return (*new, torch.empty(lib.kvc_verify_workspace_bytes(step._at, vocab), dtype=torch.uint8,
                                      device=parents.device) if workspace is None else workspace)
        path, counts, chosen, workspace = _allocate(stream, missing)
    packed = _pack_draft(vocab, children, _plain(parents, torch.int32, (N,), "parents"),
                         _plain(tokens, torch.int32, (N,), "tokens"), *_pack_probabilities(target, N, vocab, "target"),
                         *_pack_probabilities(draft, N, vocab, "draft"),
                         _plain(uniforms, torch.float32, (N,), "uniforms"), _plain(last, torch.float32, (n,), "last"),
                         _plain(path, torch.int32, (N,), "path"), _plain(counts, torch.int32, (n,), "counts"),
                         _plain(chosen, torch.int32, (n,), "chosen"))
    status = lib.kvc_verify(step._at, packed, workspace.data_ptr(), workspace.numel() * workspace.element_size(), raw)
    if status:
        raise KvcError(status, "kvc_verify")
    return path, counts, chosen


def kvc_keep(cache: Cache, step: Step, path: torch.Tensor, counts: torch.Tensor, layer_begin: int = 0,
             layer_end: Optional[int] = None, stream=None) -> None:
    """Brings the rows of each sequence's accepted tokens (kvc_verify's path and counts) to the first of its new tokens'
    places in the cache."""
    raw = _raw_stream(stream, cache, step, path, counts)
    status = load().kvc_keep(cache._at, cache._scales_at, step._at, _plain(path, torch.int32, (step.num_rows,), "path"),
                             _plain(counts, torch.int32, (step.contexts.numel(),), "counts"), layer_begin,
                             cache._layers if layer_end is None else layer_end, raw)
    if status:
        raise KvcError(status, "kvc_keep")
