"""Incremental chunked-prefill attention over a paged KV cache, for AMD MI355X (gfx950).

Python binding of the C ABI in ``include/s2l.h`` (libs2l.so, built from ``csrc/``).  The
functions below carry the C names and only marshal arguments: torch tensors supply device
memory and streams, every step of the computation runs in the library's HIP kernels.

Typical step for one layer (Stream2LLM append mode: a chunk of C tokens arrives for a
request that already holds P cached tokens)::

    batch = Batch(prefix_lens, chunk_lens, block_tables)       # P_r, C_r, page ids
    s2l_kv_append(cache, batch, k_new, v_new)                  # pages <- chunk K/V
    ws = torch.empty(s2l_attn_workspace_bytes(batch, Hq, Hkv), dtype=torch.uint8, device="cuda")
    plan = s2l_attn_plan(batch, Hq, Hkv, ws)                   # once per step, all layers
    s2l_chunk_prefill_attn(cache, batch, q, Hq, 128 ** -0.5, out, lse, plan, ws)

Where queries and keys come unrotated from the projection, ``s2l_rope_kv_append`` takes the place of
the append and rotates them on the way (positions of one axis or several, ``Rope``).  A layer of linear
attention keeps a state a request instead of pages (``LinearState``)::

    s2l_rope_kv_append(cache, batch, rope, q_raw, q, k_raw, v)     # pages <- rotated K, V; q <- rotated Q
    s2l_rope_qk(batch, rope, q_raw, q, k_raw, k)                   # a layer without pages
    ws = torch.empty(s2l_linear_attn_workspace_bytes(batch, Hq), dtype=torch.uint8, device="cuda")
    s2l_linear_attn(state, batch, q, k, v, 128 ** -0.5, out, ws)

Where the model norms queries and keys for each head before they rotate, ``s2l_norm_rope_kv_append`` and
``s2l_norm_rope_qk`` do both in the rotation's launch (``QKNorm``).  A cache may be held in 4 bits: pools of
``MXFP4_RUN_BYTES`` bytes a page and head, which every call on a cache takes as it takes the others (not the
attention with quantised queries); ``s2l_kv_read`` reads any cache's rows back as bf16 values::

    pools = [torch.zeros((pages, Hkv, MXFP4_RUN_BYTES), dtype=torch.uint8, device="cuda") for _ in "kv"]
    cache = PagedKVCache(*pools)
    s2l_norm_rope_kv_append(cache, batch, QKNorm(q_weight, k_weight), rope, q_raw, q, k_raw, v)
    s2l_kv_read(cache, batch, S2L_READ_CHUNK, batch.cu_chunk, k_rows, v_rows)
"""
import contextlib
import ctypes

import numpy as np
import torch

from . import _lib
from ._lib import (S2L_KV_BF16, S2L_KV_FP8_E4M3, S2L_KV_MXFP4, S2L_READ_ALL, S2L_READ_CHUNK, S2L_READ_PREFIX, S2LError,
                   S2LLibraryMissing, s2l_plan_info, s2l_plan_opts)

__all__ = ["PagedKVCache", "Batch", "Rope", "QKNorm", "LinearState", "rope_pair_axes", "plan_opts", "S2LError", "S2LLibraryMissing",
           "s2l_abi_version", "s2l_kv_append", "s2l_kv_gather", "s2l_kv_swap_out", "s2l_kv_swap_in",
           "s2l_kv_read", "S2L_READ_PREFIX", "S2L_READ_ALL", "S2L_READ_CHUNK", "MXFP4_RUN_BYTES",
           "s2l_rope_qk", "s2l_rope_kv_append", "s2l_norm_rope_qk", "s2l_norm_rope_kv_append", "s2l_linear_attn", "s2l_linear_attn_workspace_bytes",
           "s2l_check_tables", "s2l_append_chunk_prefill_attn", "s2l_calib_stream_read", "s2l_calib_mfma_bf16", "s2l_attn_workspace_bytes",
           "s2l_attn_plan", "s2l_chunk_prefill_attn", "s2l_chunk_prefill_attn_q8", "s2l_attn_main", "s2l_split_reduce",
           "s2l_plan_host", "library_path", "plan_status", "s2l_chunk_prefill_attn_noalloc"]

HEAD_DIM = 128
PAGE_SIZE = 16
MXFP4_RUN_BYTES = _lib.S2L_MXFP4_RUN_BYTES     # of one page of one kv head: 16 x 64 of codes, 16 x 4 of scales


def library_path():
    return _lib.LIB_PATH


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    return ctypes.c_void_p(int(stream))


def _check(t, dtype, name):
    if t is None:
        return
    if t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor (got {t.dtype}, "
                         f"contiguous={t.is_contiguous()})")


class PagedKVCache:
    """One layer's K and V page pools, each [num_pages][Hkv][16][128] (bf16, or uint8 E4M3), or
    [num_pages][Hkv][MXFP4_RUN_BYTES] uint8 (MXFP4: codes and their scales, no scales apart)."""

    def __init__(self, k_pages, v_pages, k_scale=None, v_scale=None):
        mxfp4 = k_pages.dtype == torch.uint8 and k_pages.dim() == 3
        fp8 = k_pages.dtype == torch.uint8 and not mxfp4
        _check(k_pages, torch.uint8 if fp8 or mxfp4 else torch.bfloat16, "k_pages")
        _check(v_pages, k_pages.dtype, "v_pages")
        if fp8:
            _check(k_scale, torch.float32, "k_scale")
            _check(v_scale, torch.float32, "v_scale")
        if mxfp4 and (k_scale is not None or v_scale is not None):
            raise ValueError("MXFP4 pools hold their scales: k_scale and v_scale must be None")
        self.k_pages, self.v_pages = k_pages, v_pages
        self.k_scale, self.v_scale = k_scale, v_scale
        self.fp8, self.mxfp4 = fp8, mxfp4
        if mxfp4:
            self._check_runs()

    def _check_runs(self):
        k, v = self.k_pages, self.v_pages
        if (k.dim() != 3 or k.shape[2] != MXFP4_RUN_BYTES or v.shape != k.shape or k.dtype != torch.uint8 or v.dtype != torch.uint8
                or not k.is_contiguous() or not v.is_contiguous()):
            raise ValueError(f"MXFP4 pools must be contiguous uint8 [num_pages][Hkv][{MXFP4_RUN_BYTES}] of one shape (got "
                             f"{k.dtype} {tuple(k.shape)}, strides {k.stride()}, and {v.dtype} {tuple(v.shape)}, strides {v.stride()})")

    @property
    def num_pages(self):
        return self.k_pages.shape[0]

    @property
    def num_kv_heads(self):
        return self.k_pages.shape[1]

    def c(self):
        if self.mxfp4:
            self._check_runs()     # the attributes may be others by now
        return _lib.s2l_kv_cache(
            k_pages=self.k_pages.data_ptr(), v_pages=self.v_pages.data_ptr(),
            k_scale=self.k_scale.data_ptr() if self.fp8 else None,
            v_scale=self.v_scale.data_ptr() if self.fp8 else None,
            num_pages=self.k_pages.shape[0], num_kv_heads=self.k_pages.shape[1],
            head_dim=HEAD_DIM if self.mxfp4 else self.k_pages.shape[3], page_size=PAGE_SIZE if self.mxfp4 else self.k_pages.shape[2],
            dtype=S2L_KV_MXFP4 if self.mxfp4 else S2L_KV_FP8_E4M3 if self.fp8 else S2L_KV_BF16)


class Batch:
    """A step's varlen batch: device length/table arrays plus the host length copies."""

    def __init__(self, prefix_lens, chunk_lens, block_tables, device="cuda"):
        self.prefix_host = np.ascontiguousarray(prefix_lens, dtype=np.int32)
        self.chunk_host = np.ascontiguousarray(chunk_lens, dtype=np.int32)
        cu = np.zeros(len(self.chunk_host) + 1, dtype=np.int32)
        cu[1:] = np.cumsum(self.chunk_host)
        self.cu_host = cu
        bt = np.ascontiguousarray(block_tables, dtype=np.int32)
        if bt.ndim == 1:
            bt = bt.reshape(len(self.prefix_host), -1)
        self.tables_host = bt
        self.prefix_lens = torch.from_numpy(self.prefix_host).to(device)
        self.chunk_lens = torch.from_numpy(self.chunk_host).to(device)
        self.cu_chunk = torch.from_numpy(cu).to(device)
        self.block_tables = torch.from_numpy(bt).to(device)

    @property
    def num_reqs(self):
        return len(self.prefix_host)

    @property
    def total_tokens(self):
        return int(self.cu_host[-1])

    def c(self):
        return _lib.s2l_batch(
            num_reqs=self.num_reqs, max_pages_per_req=self.tables_host.shape[1],
            prefix_lens=self.prefix_lens.data_ptr(), chunk_lens=self.chunk_lens.data_ptr(),
            cu_chunk=self.cu_chunk.data_ptr(), block_tables=self.block_tables.data_ptr(),
            prefix_lens_host=self.prefix_host.ctypes.data_as(_lib.P_i32),
            chunk_lens_host=self.chunk_host.ctypes.data_as(_lib.P_i32))


def rope_pair_axes(sections, cyclic=False):
    """The position axis of each rotated pair, for `sections[a]` pairs turning by axis a: the axes in
    blocks one after another, or (cyclic) in turn: axis a > 0 takes pairs a, a + n, a + 2 n, ... until
    it has its number, axis 0 the rest."""
    sections = [int(m) for m in sections]
    if not sections or min(sections) < 0:
        raise ValueError(f"sections must be counts of pairs (got {sections})")
    n, pairs = len(sections), sum(sections)
    if not cyclic:
        return [a for a, m in enumerate(sections) for _ in range(m)]
    axes = [i % n if i // n < sections[i % n] else 0 for i in range(pairs)]
    if [axes.count(a) for a in range(n)] != sections:
        raise ValueError(f"sections {sections} do not fit in turns over {pairs} pairs")
    return axes


class Rope:
    """How rows rotate: pair i of a head turns by (its axis's position) * inv_freq[i].

    inv_freq: device fp32 [rot_dim / 2].  positions: None (row i of request r is at P_r + i), or a
    device int32 tensor [T] or [axes][T], one position per row of the batch and axis.  pair_axes: the
    axis of each pair (``rope_pair_axes``), None for axis 0 throughout.  adjacent: pairs are dims
    (2 i, 2 i + 1) instead of (i, i + rot_dim / 2).  scale: a factor on the rotated dims."""

    def __init__(self, inv_freq, positions=None, pair_axes=None, adjacent=False, scale=1.0):
        self.inv_freq = inv_freq
        self._check_freq()
        pair_axes = [0] * inv_freq.shape[0] if pair_axes is None else [int(a) for a in pair_axes]
        if len(pair_axes) != inv_freq.shape[0] or min(pair_axes) < 0 or max(pair_axes) >= _lib.S2L_ROPE_MAX_AXES:
            raise ValueError(f"pair_axes must name an axis below {_lib.S2L_ROPE_MAX_AXES} for each of the "
                             f"{inv_freq.shape[0]} pairs")
        self.positions, self.adjacent, self.scale = positions, bool(adjacent), float(scale)
        self.pair_axis = bytes(pair_axes) + bytes(64 - len(pair_axes))

    def _check_freq(self):
        _check(self.inv_freq, torch.float32, "inv_freq")
        if self.inv_freq.dim() != 1 or not 1 <= self.inv_freq.shape[0] <= HEAD_DIM // 2:
            raise ValueError(f"inv_freq must be a vector of 1 to {HEAD_DIM // 2} pairs")

    def c(self, total_tokens, device):
        self._check_freq()       # the attribute may be another by now
        p = self.positions
        if p is not None and (p.dtype != torch.int32 or p.dim() not in (1, 2) or p.stride(-1) != 1 and p.shape[-1] > 1
                              or p.shape[-1] < total_tokens or p.dim() == 2 and p.shape[0] > 1 and p.stride(0) < 0):
            raise ValueError(f"positions must be an int32 tensor [T] or [axes][T] of {total_tokens} rows, each axis contiguous")
        for t, name in ((self.inv_freq, "inv_freq"), (p, "positions")):
            if t is not None and t.device != device:
                raise ValueError(f"{name} is on {t.device}, the batch on {device}")
        return _lib.s2l_rope(inv_freq=self.inv_freq.data_ptr(), positions=None if p is None else p.data_ptr(),
                             pos_stride=0 if p is None or p.dim() == 1 else p.stride(0), rot_dim=2 * self.inv_freq.shape[0],
                             num_axes=1 if p is None or p.dim() == 1 else p.shape[0],
                             flags=_lib.S2L_ROPE_ADJACENT if self.adjacent else 0, scale=self.scale,
                             pair_axis=(ctypes.c_uint8 * 64)(*self.pair_axis))


class QKNorm:
    """The norms of queries and keys for each head: x / sqrt(mean x^2 + eps) * (weight + offset).

    q_weight, k_weight: device [128], both bf16 or both fp32; None: no weight (nor offset).  offset: 1 where
    weights are kept as their distance from one.  eps: at least 2^-126 (what is less is zero to the hardware's root)."""

    def __init__(self, q_weight=None, k_weight=None, eps=1e-6, offset=0.0):
        self.q_weight, self.k_weight, self.eps, self.offset = q_weight, k_weight, float(eps), float(offset)
        self._check_weights()

    def _check_weights(self):
        given = [(w, n) for w, n in ((self.q_weight, "q_weight"), (self.k_weight, "k_weight")) if w is not None]
        for w, name in given:
            _check(w, torch.float32 if w.dtype == torch.float32 else torch.bfloat16, name)
            if tuple(w.shape) != (HEAD_DIM,) or w.dtype != given[0][0].dtype:
                raise ValueError(f"{name} must be a vector of {HEAD_DIM}, of one type with the other (got {w.dtype}, shape {tuple(w.shape)})")
        return given

    def c(self, device):
        given = self._check_weights()     # the attributes may be others by now
        for w, name in given:
            if w.device != device:
                raise ValueError(f"{name} is on {w.device}, the batch on {device}")
        return _lib.s2l_qk_norm(q_weight=None if self.q_weight is None else self.q_weight.data_ptr(),
                                k_weight=None if self.k_weight is None else self.k_weight.data_ptr(), eps=self.eps, offset=self.offset,
                                weight_dtype=_lib.S2L_NORM_FP32 if given and given[0][0].dtype == torch.float32 else _lib.S2L_NORM_BF16)


class LinearState:
    """A linear attention layer's request states: states fp32 [slots][Hq][128][128], log_decay fp32
    [Hq] (ln of each head's decay, <= 0), and each request's slots, int32 [R]: slot_in (-1: a zero
    state) is read, slot_out (-1: not kept) is written; the same slot advances in place.  Slots are the
    caller's: the scheduler and the swap calls move pages alone, a preempted request's state stays in its slot."""

    def __init__(self, states, log_decay, slot_in, slot_out):
        self.states, self.log_decay, self.slot_in, self.slot_out = states, log_decay, slot_in, slot_out
        self._check_states()

    def _check_states(self):
        _check(self.states, torch.float32, "states")
        _check(self.log_decay, torch.float32, "log_decay")
        if self.states.dim() != 4 or tuple(self.states.shape[2:]) != (HEAD_DIM, HEAD_DIM) or self.log_decay.shape != self.states.shape[1:2]:
            raise ValueError(f"states must be [slots][Hq][{HEAD_DIM}][{HEAD_DIM}] and log_decay [Hq]")

    @property
    def num_heads(self):
        return self.states.shape[1]

    def c(self, num_reqs, device):
        self._check_states()     # the attributes may be others by now
        for t, name in ((self.slot_in, "slot_in"), (self.slot_out, "slot_out")):
            _check(t, torch.int32, name)
            if t.dim() != 1 or t.shape[0] != num_reqs:
                raise ValueError(f"{name} must hold one slot for each of the {num_reqs} requests")
        for t, name in ((self.states, "states"), (self.log_decay, "log_decay"), (self.slot_in, "slot_in"), (self.slot_out, "slot_out")):
            if t.device != device:
                raise ValueError(f"{name} is on {t.device}, the batch on {device}")
        return _lib.s2l_linear_state(states=self.states.data_ptr(), log_decay=self.log_decay.data_ptr(),
                                     slot_in=self.slot_in.data_ptr(), slot_out=self.slot_out.data_ptr(),
                                     num_slots=self.states.shape[0], num_heads=self.states.shape[1])


def plan_opts(target_items=0, min_split_keys=0, max_splits=0, tile_cols=0, key_halves=0):
    return s2l_plan_opts(target_items=target_items, min_split_keys=min_split_keys,
                         max_splits=max_splits, tile_cols=tile_cols, key_halves=key_halves)


def _opts_ptr(opts):
    return None if opts is None else ctypes.byref(opts)


def s2l_abi_version():
    return _lib.lib().s2l_abi_version()


_native = None


def _load_native():
    """The native marshalling of the calls that every step makes.  Its functions return None for
    arguments that are not of the plain form it expects; the ctypes path then takes them (or says
    what is wrong with them)."""
    global _native
    if _native is None:
        # a torch without GPU support lacks the last two: no current stream, so the ctypes path
        device, raw_stream = (getattr(torch._C, n, None) for n in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))
        _native = _lib.binding((torch.Tensor, PagedKVCache, Batch, s2l_plan_opts, s2l_plan_info, torch.cuda.Stream,
                                torch.bfloat16, torch.float32, torch.uint8, torch.cuda.is_initialized, device, raw_stream,
                                Rope, LinearState, torch.int32, QKNorm, torch.nn.Parameter))
    return _native


def s2l_kv_append(cache, batch, k_new, v_new, stream=None):
    st = (_native or _load_native()).append(cache, batch, k_new, v_new, stream)
    if st is not None:
        return _lib.failed("s2l_kv_append", st) if st else None
    _check(k_new, torch.bfloat16, "k_new")
    _check(v_new, torch.bfloat16, "v_new")
    cc, bc = cache.c(), batch.c()
    _lib.call("s2l_kv_append", ctypes.byref(cc), ctypes.byref(bc), _ptr(k_new), _ptr(v_new), _stream(stream))


def _rows(t, name, batch):
    """(pointer, row stride, heads) of a device bf16 tensor [rows][heads][128], rows anywhere apart,
    that holds the batch's rows."""
    if t.dtype != torch.bfloat16 or t.dim() != 3 or t.shape[2] != HEAD_DIM or t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != HEAD_DIM):
        raise ValueError(f"{name} must be bf16 rows [T][heads][{HEAD_DIM}] of contiguous heads (got {t.dtype}, shape "
                         f"{tuple(t.shape)}, strides {t.stride()})")
    if t.shape[0] < batch.total_tokens:
        raise ValueError(f"{name} has {t.shape[0]} rows, the batch {batch.total_tokens}")
    if not t.is_cuda or t.device != batch.chunk_lens.device:
        raise ValueError(f"{name} is on {t.device}, the batch on {batch.chunk_lens.device}")
    return _ptr(t), t.stride(0), t.shape[1]


def _call_on(batch, name, *args, stream):
    """An entry point's call with the batch's device current: `stream` (None: that device's current
    stream) is one of its streams."""
    with torch.cuda.device(batch.chunk_lens.device):
        _lib.call(name, *args, _stream(stream))


def _same_heads(a, b, what):
    if a != b:
        raise ValueError(f"{what} differ in their heads ({a} and {b})")


def _rotate(name, batch, norm, rope, q, q_out, k, k_out, stream):
    """s2l_rope_qk, or s2l_norm_rope_qk with a norm."""
    qp, qs, hq = _rows(q, "q", batch)
    op, os_, ho = _rows(q_out, "q_out", batch)
    _same_heads(hq, ho, "q and q_out")
    kp, ks, hkv, kop, kos = None, 0, 0, None, 0
    if k is not None:
        kp, ks, hkv = _rows(k, "k", batch)
        kop, kos, ho = _rows(k_out, "k_out", batch)
        _same_heads(hkv, ho, "k and k_out")
    device = batch.chunk_lens.device
    bc, rc = batch.c(), rope.c(batch.total_tokens, device)
    how = [ctypes.byref(rc)] if norm is None else [ctypes.byref(norm.c(device)), ctypes.byref(rc)]
    _call_on(batch, name, ctypes.byref(bc), *how, qp, qs, hq, op, os_, kp, ks, hkv, kop, kos, stream=stream)


def _rotate_append(name, cache, batch, norm, rope, q, q_out, k, v, stream):
    """s2l_rope_kv_append, or s2l_norm_rope_kv_append with a norm."""
    qp, qs, hq, op, os_ = None, 0, 0, None, 0
    if q is not None:
        qp, qs, hq = _rows(q, "q", batch)
        op, os_, ho = _rows(q_out, "q_out", batch)
        _same_heads(hq, ho, "q and q_out")
    kp, ks, hk = _rows(k, "k", batch)
    vp, vs, hv = _rows(v, "v", batch)
    _same_heads(hk, cache.num_kv_heads, "k and the cache")
    _same_heads(hv, cache.num_kv_heads, "v and the cache")
    _cache_device(cache, batch)
    device = batch.chunk_lens.device
    cc, bc, rc = cache.c(), batch.c(), rope.c(batch.total_tokens, device)
    how = [ctypes.byref(rc)] if norm is None else [ctypes.byref(norm.c(device)), ctypes.byref(rc)]
    _call_on(batch, name, ctypes.byref(cc), ctypes.byref(bc), *how, qp, qs, hq, op, os_, kp, ks, vp, vs, stream=stream)


def _cache_device(cache, batch):
    for name in ("k_pages", "v_pages", "k_scale", "v_scale") if cache.fp8 else ("k_pages", "v_pages"):
        if getattr(cache, name).device != batch.chunk_lens.device:
            raise ValueError(f"{name} is on {getattr(cache, name).device}, the batch on {batch.chunk_lens.device}")


def s2l_rope_qk(batch, rope, q, q_out, k=None, k_out=None, stream=None):
    """Rotate the batch's query rows q into q_out and its key rows k (if any) into k_out: bf16
    [rows][heads][128], rows at any stride; an output may be its own input."""
    st = (_native or _load_native()).rope_qk(batch, rope, q, q_out, k, k_out, stream)
    if st is not None:
        return _lib.failed("s2l_rope_qk", st) if st else None
    _rotate("s2l_rope_qk", batch, None, rope, q, q_out, k, k_out, stream)


def s2l_rope_kv_append(cache, batch, rope, q, q_out, k, v, stream=None):
    """s2l_kv_append of the rotated keys and of the values, with the rotated queries in q_out (q and
    q_out None: none), in one launch; tensors as for s2l_rope_qk."""
    st = (_native or _load_native()).rope_append(cache, batch, rope, q, q_out, k, v, stream)
    if st is not None:
        return _lib.failed("s2l_rope_kv_append", st) if st else None
    _rotate_append("s2l_rope_kv_append", cache, batch, None, rope, q, q_out, k, v, stream)


def _need_norm(norm):
    if not isinstance(norm, QKNorm):
        raise ValueError(f"norm must be a QKNorm (got {type(norm).__name__})")


def s2l_norm_rope_qk(batch, norm, rope, q, q_out, k=None, k_out=None, stream=None):
    """s2l_rope_qk of queries and keys that `norm` (a QKNorm) norms for each head first."""
    st = (_native or _load_native()).norm_rope_qk(batch, norm, rope, q, q_out, k, k_out, stream)
    if st is not None:
        return _lib.failed("s2l_norm_rope_qk", st) if st else None
    _need_norm(norm)
    _rotate("s2l_norm_rope_qk", batch, norm, rope, q, q_out, k, k_out, stream)


def s2l_norm_rope_kv_append(cache, batch, norm, rope, q, q_out, k, v, stream=None):
    """s2l_rope_kv_append of queries and keys that `norm` (a QKNorm) norms for each head first."""
    st = (_native or _load_native()).norm_rope_append(cache, batch, norm, rope, q, q_out, k, v, stream)
    if st is not None:
        return _lib.failed("s2l_norm_rope_kv_append", st) if st else None
    _need_norm(norm)
    _rotate_append("s2l_norm_rope_kv_append", cache, batch, norm, rope, q, q_out, k, v, stream)


def s2l_linear_attn_workspace_bytes(batch, num_q_heads):
    """Workspace bytes of the batch's s2l_linear_attn, which cuts chunks by the CUs of the batch's device."""
    bc = batch.c()
    n = ctypes.c_size_t(0)
    device = batch.chunk_lens.device
    with torch.cuda.device(device) if device.type == "cuda" else contextlib.nullcontext():
        _lib.call("s2l_linear_attn_workspace_bytes", ctypes.byref(bc), num_q_heads, ctypes.byref(n))
    return n.value


def s2l_linear_attn(state, batch, q, k, v, scale, out, workspace=None, stream=None):
    """Linear attention of the batch's chunks over `state` (advanced from its slot_in to its slot_out):
    out[i][h] = scale * q_i[h] S after S <- exp(log_decay[h]) S + k_i v_i^T; tensors as for
    s2l_rope_qk, the workspace a device uint8 tensor (None where no bytes are needed)."""
    st = (_native or _load_native()).linear(state, batch, q, k, v, scale, out, workspace, stream)
    if st is not None:
        return _lib.failed("s2l_linear_attn", st) if st else None
    qp, qs, hq = _rows(q, "q", batch)
    kp, ks, hkv = _rows(k, "k", batch)
    vp, vs, hv = _rows(v, "v", batch)
    op, os_, ho = _rows(out, "out", batch)
    _same_heads(hq, state.num_heads, "q and the state")
    _same_heads(hq, ho, "q and out")
    _same_heads(hkv, hv, "k and v")
    if workspace is not None:
        _check(workspace, torch.uint8, "workspace")
        if workspace.device != batch.chunk_lens.device:
            raise ValueError(f"workspace is on {workspace.device}, the batch on {batch.chunk_lens.device}")
    bc, sc = batch.c(), state.c(batch.num_reqs, batch.chunk_lens.device)
    _call_on(batch, "s2l_linear_attn", ctypes.byref(sc), ctypes.byref(bc), qp, qs, kp, ks, vp, vs, hkv, float(scale), op, os_,
             _ptr(workspace), 0 if workspace is None else workspace.numel(), stream=stream)


def _swap(name, cache, pairs, host_k, host_v, stream):
    if host_k.is_cuda or host_v.is_cuda or host_k.dtype != cache.k_pages.dtype or host_v.dtype != host_k.dtype:
        raise ValueError("host pools must be host tensors of the cache's element type")
    if not (host_k.is_contiguous() and host_v.is_contiguous()) or host_k.shape != host_v.shape:
        raise ValueError("host pools must be contiguous and of one shape")
    if host_k.dim() < 1 or host_k.numel() * cache.num_pages != cache.k_pages.numel() * host_k.shape[0]:
        raise ValueError(f"host pools must hold pages of the cache's size ({tuple(cache.k_pages.shape[1:])}, got {tuple(host_k.shape)})")
    _check(pairs, torch.int32, "pairs")
    if pairs.dim() != 2 or pairs.shape[1] != 2 or not pairs.is_cuda:
        raise ValueError("pairs must be a device int32 tensor [n][2]")
    cc = cache.c()
    _lib.call(name, ctypes.byref(cc), _ptr(pairs), pairs.shape[0], _ptr(host_k), _ptr(host_v),
              host_k.shape[0], _stream(stream))


def s2l_kv_swap_out(cache, pairs, host_k, host_v, stream=None):
    """Device pages pairs[i][0] -> pinned host pages pairs[i][1] (K and V)."""
    _swap("s2l_kv_swap_out", cache, pairs, host_k, host_v, stream)


def s2l_kv_swap_in(cache, pairs, host_k, host_v, stream=None):
    """Pinned host pages pairs[i][0] -> device pages pairs[i][1] (K and V)."""
    _swap("s2l_kv_swap_in", cache, pairs, host_k, host_v, stream)


def s2l_check_tables(cache, batch, counts, stream=None):
    """Count used block-table entries outside the pool into the device int32[2] `counts`."""
    _check(counts, torch.int32, "counts")
    cc, bc = cache.c(), batch.c()
    _lib.call("s2l_check_tables", ctypes.byref(cc), ctypes.byref(bc), _ptr(counts), _stream(stream))


def s2l_calib_stream_read(buf, sink, grid, stream=None):
    """One streaming read of the device tensor `buf` (measurement support)."""
    _lib.call("s2l_calib_stream_read", _ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), int(grid),
              _stream(stream))


def s2l_calib_mfma_bf16(iters, sink, grid, stream=None):
    """A register-only bf16 MFMA loop (measurement support); returns its flop count."""
    flops = ctypes.c_int64()
    _lib.call("s2l_calib_mfma_bf16", int(iters), _ptr(sink), int(grid), ctypes.byref(flops), _stream(stream))
    return flops.value


def s2l_kv_gather(cache, batch, include_chunk, cu_out, k_out, v_out, stream=None):
    _check(cu_out, torch.int32, "cu_out")
    cc, bc = cache.c(), batch.c()
    _lib.call("s2l_kv_gather", ctypes.byref(cc), ctypes.byref(bc), int(include_chunk), _ptr(cu_out),
              _ptr(k_out), _ptr(v_out), _stream(stream))


def s2l_kv_read(cache, batch, part, cu_out, k_out, v_out, stream=None):
    """Read cached K/V back as bf16 values: position number i of request r's part (S2L_READ_PREFIX, _ALL or
    _CHUNK) goes to row cu_out[r] + i of k_out and v_out, contiguous bf16 [rows][Hkv][128]; rows that they
    do not have are not written.  cu_out: device int32, a row for each request (batch.cu_chunk for chunks)."""
    st = (_native or _load_native()).read(cache, batch, part, cu_out, k_out, v_out, stream)
    if st is not None:
        return _lib.failed("s2l_kv_read", st) if st else None
    _check(cu_out, torch.int32, "cu_out")
    if cu_out.dim() != 1 or cu_out.shape[0] < batch.num_reqs:
        raise ValueError(f"cu_out must hold a row for each of the {batch.num_reqs} requests")
    for t, name in ((k_out, "k_out"), (v_out, "v_out")):
        _check(t, torch.bfloat16, name)
        if t.dim() != 3 or t.shape[1] != cache.num_kv_heads or t.shape[2] != HEAD_DIM or t.shape[0] != k_out.shape[0]:
            raise ValueError(f"{name} must be [rows][{cache.num_kv_heads}][{HEAD_DIM}], of as many rows as the other (got {tuple(t.shape)})")
    for t, name in ((cu_out, "cu_out"), (k_out, "k_out"), (v_out, "v_out")):
        if t.device != batch.chunk_lens.device:
            raise ValueError(f"{name} is on {t.device}, the batch on {batch.chunk_lens.device}")
    _cache_device(cache, batch)
    cc, bc = cache.c(), batch.c()
    _call_on(batch, "s2l_kv_read", ctypes.byref(cc), ctypes.byref(bc), int(part), _ptr(cu_out), _ptr(k_out), _ptr(v_out),
             k_out.shape[0], stream=stream)


def s2l_attn_workspace_bytes(batch, num_q_heads, num_kv_heads, opts=None):
    bc = batch.c()
    n = ctypes.c_size_t(0)
    _lib.call("s2l_attn_workspace_bytes", ctypes.byref(bc), num_q_heads, num_kv_heads, _opts_ptr(opts),
              ctypes.byref(n))
    return n.value


def s2l_attn_plan(batch, num_q_heads, num_kv_heads, workspace, opts=None, stream=None):
    info = s2l_plan_info()
    st = (_native or _load_native()).plan(batch, num_q_heads, num_kv_heads, opts, workspace, info, stream)
    if st is not None:
        return _lib.failed("s2l_attn_plan", st) if st else info
    _check(workspace, torch.uint8, "workspace")
    bc = batch.c()
    _lib.call("s2l_attn_plan", ctypes.byref(bc), num_q_heads, num_kv_heads, _opts_ptr(opts),
              _ptr(workspace), workspace.numel(), ctypes.byref(info), _stream(stream))
    return info


PLAN_STATUS_OFFSET = 36      # S2L_PLAN_STATUS_OFFSET of include/s2l.h


def plan_status(workspace):
    """The plan's int32 status word in `workspace` (a device uint8 tensor that s2l_attn_plan
    filled), as a 0-dim device tensor: 0 = planned, 1 = the device length arrays needed more
    than the host copies planned for (the attention calls then write NaN and compute
    nothing).  Read it after the stream has passed the plan."""
    _check(workspace, torch.uint8, "workspace")
    return workspace[PLAN_STATUS_OFFSET:PLAN_STATUS_OFFSET + 4].view(torch.int32)[0]


_ATTN = {"s2l_chunk_prefill_attn": 0, "s2l_chunk_prefill_attn_q8": 1, "s2l_attn_main": 2}


def _attn(name, cache, batch, q, num_q_heads, softmax_scale, out, lse, plan, workspace, stream):
    st = (_native or _load_native()).attn(_ATTN[name], cache, batch, q, num_q_heads, softmax_scale, out, lse, plan,
                                      workspace, stream)
    if st is not None:
        return _lib.failed(name, st) if st else None
    _check(q, torch.bfloat16, "q")
    _check(out, torch.bfloat16, "out")
    _check(lse, torch.float32, "lse")
    _check(workspace, torch.uint8, "workspace")
    cc, bc = cache.c(), batch.c()
    _lib.call(name, ctypes.byref(cc), ctypes.byref(bc), _ptr(q), num_q_heads, float(softmax_scale),
              _ptr(out), _ptr(lse), ctypes.byref(plan), _ptr(workspace), workspace.numel(), _stream(stream))


def s2l_chunk_prefill_attn(cache, batch, q, num_q_heads, softmax_scale, out, lse, plan, workspace,
                           stream=None):
    _attn("s2l_chunk_prefill_attn", cache, batch, q, num_q_heads, softmax_scale, out, lse, plan,
          workspace, stream)


def s2l_chunk_prefill_attn_q8(cache, batch, q, num_q_heads, softmax_scale, out, lse, plan, workspace,
                              stream=None):
    """s2l_chunk_prefill_attn with Q quantised to e4m3 per (token, head) row and Q K^T on the
    fp8 MFMA (e4m3 caches only)."""
    _attn("s2l_chunk_prefill_attn_q8", cache, batch, q, num_q_heads, softmax_scale, out, lse, plan,
          workspace, stream)


def s2l_append_chunk_prefill_attn(cache, batch, k_new, v_new, q, num_q_heads, softmax_scale, out, lse, plan,
                                  workspace, stream=None):
    """s2l_kv_append + s2l_chunk_prefill_attn, in one attention launch where possible;
    returns True when the single launch was used."""
    r = (_native or _load_native()).fused(cache, batch, q, num_q_heads, softmax_scale, out, lse, plan, workspace, stream,
                                      k_new, v_new)
    if r is not None:
        return _lib.failed("s2l_append_chunk_prefill_attn", r[0]) if r[0] else r[1]
    for t, n in ((k_new, "k_new"), (v_new, "v_new"), (q, "q"), (out, "out")):
        _check(t, torch.bfloat16, n)
    _check(lse, torch.float32, "lse")
    _check(workspace, torch.uint8, "workspace")
    cc, bc = cache.c(), batch.c()
    fused = ctypes.c_int32()
    _lib.call("s2l_append_chunk_prefill_attn", ctypes.byref(cc), ctypes.byref(bc), _ptr(k_new), _ptr(v_new),
              _ptr(q), num_q_heads, float(softmax_scale), _ptr(out), _ptr(lse), ctypes.byref(plan),
              _ptr(workspace), workspace.numel(), ctypes.byref(fused), _stream(stream))
    return bool(fused.value)


NOALLOC_SCRATCH_BYTES = 64 << 20     # S2L_NOALLOC_SCRATCH_BYTES of include/s2l.h


def s2l_chunk_prefill_attn_noalloc(cache, batch, q, num_q_heads, softmax_scale, out, lse, opts=None, stream=None):
    """Plan + attention + merge with the library's own scratch (no workspace, no allocation);
    returns the plan's s2l_plan_info.  Calls overlapping on one GPU race (shared scratch)."""
    _check(q, torch.bfloat16, "q")
    _check(out, torch.bfloat16, "out")
    _check(lse, torch.float32, "lse")
    info = s2l_plan_info()
    cc, bc = cache.c(), batch.c()
    _lib.call("s2l_chunk_prefill_attn_noalloc", ctypes.byref(cc), ctypes.byref(bc), _ptr(q), num_q_heads,
              float(softmax_scale), _ptr(out), _ptr(lse), _opts_ptr(opts), ctypes.byref(info), _stream(stream))
    return info


def s2l_attn_main(cache, batch, q, num_q_heads, softmax_scale, out, lse, plan, workspace, stream=None):
    _attn("s2l_attn_main", cache, batch, q, num_q_heads, softmax_scale, out, lse, plan, workspace, stream)


def s2l_split_reduce(batch, num_q_heads, out, lse, plan, workspace, stream=None):
    st = (_native or _load_native()).reduce(batch, num_q_heads, out, lse, plan, workspace, stream)
    if st is not None:
        return _lib.failed("s2l_split_reduce", st) if st else None
    _check(out, torch.bfloat16, "out")
    _check(lse, torch.float32, "lse")
    bc = batch.c()
    _lib.call("s2l_split_reduce", ctypes.byref(bc), num_q_heads, _ptr(out), _ptr(lse), ctypes.byref(plan),
              _ptr(workspace), workspace.numel(), _stream(stream))


def s2l_plan_host(prefix_lens, chunk_lens, num_q_heads, num_kv_heads, opts=None, num_cus=256,
                  with_items=False):
    """Host-only partition: returns (s2l_plan_info, items [num_items][8] int32 or None)."""
    P = np.ascontiguousarray(prefix_lens, dtype=np.int32)
    C = np.ascontiguousarray(chunk_lens, dtype=np.int32)
    info = s2l_plan_info()
    _lib.call("s2l_plan_host", len(P), P.ctypes.data_as(_lib.P_i32), C.ctypes.data_as(_lib.P_i32),
              num_q_heads, num_kv_heads, _opts_ptr(opts), num_cus, ctypes.byref(info), None, 0)
    if not with_items:
        return info, None
    items = np.zeros((max(info.num_items, 1), 8), dtype=np.int32)
    _lib.call("s2l_plan_host", len(P), P.ctypes.data_as(_lib.P_i32), C.ctypes.data_as(_lib.P_i32),
              num_q_heads, num_kv_heads, _opts_ptr(opts), num_cus, ctypes.byref(info),
              items.ctypes.data_as(_lib.P_i32), info.num_items)
    return info, items[:info.num_items]
