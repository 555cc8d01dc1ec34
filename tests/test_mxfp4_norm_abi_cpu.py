"""Refusals of MXFP4 caches, reading back and the normed rotation, without a GPU: every call fails the
host's checks, in the library and in the package, before anything is enqueued."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from paper_2604_16395_amd import _lib
from tests.test_abi_cpu import FAKE, _batch, _cache, _status
from tests.test_rope_linear_abi_cpu import BAD_ROPES, _rope

EINVAL, ERANGE, ENOTSUP = _lib.S2L_EINVAL, _lib.S2L_ERANGE, _lib.S2L_ENOTSUP
byref = ctypes.byref


def _norm(**kw):
    n = _lib.s2l_qk_norm(q_weight=FAKE, k_weight=FAKE, eps=1e-6, offset=0.0, weight_dtype=0)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def _qk(norm, rope, batch, q=FAKE, qs=1024, hq=8, qo=FAKE, qos=1024, k=FAKE, ks=256, hkv=2, ko=FAKE, kos=256):
    return _status("s2l_norm_rope_qk", byref(batch) if batch else None, byref(norm) if norm else None, byref(rope) if rope else None,
                   q, qs, hq, qo, qos, k, ks, hkv, ko, kos, None)


def _append(norm, rope, batch, cache, q=FAKE, qs=1024, hq=8, qo=FAKE, qos=1024, k=FAKE, ks=256, v=FAKE, vs=256):
    return _status("s2l_norm_rope_kv_append", byref(cache) if cache else None, byref(batch) if batch else None,
                   byref(norm) if norm else None, byref(rope) if rope else None, q, qs, hq, qo, qos, k, ks, v, vs, None)


def _read(cache, batch, part=1, cu=FAKE, k=FAKE, v=FAKE, rows=100):
    return _status("s2l_kv_read", byref(cache) if cache else None, byref(batch) if batch else None, part, cu, k, v, rows, None)


@pytest.mark.parametrize("dtype", [0, 2])
@pytest.mark.parametrize("kw,status", BAD_ROPES)
def test_bad_rotations(kw, status, dtype):
    b, keep = _batch([3], [4])
    for st, msg in (_qk(_norm(), _rope(**kw), b), _append(_norm(), _rope(**kw), b, _cache(dtype=dtype))):
        assert st == status and msg


@pytest.mark.parametrize("kw", [dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(offset=float("nan")),
                                dict(offset=float("inf")), dict(weight_dtype=2), dict(weight_dtype=-1), dict(q_weight=FAKE + 1),
                                dict(k_weight=FAKE + 2, weight_dtype=1)])
def test_bad_norms(kw):
    b, keep = _batch([3], [4])
    for st, msg in (_qk(_norm(**kw), _rope(), b), _append(_norm(**kw), _rope(), b, _cache())):
        assert st == EINVAL and "norm" in msg


@pytest.mark.parametrize("kw", [dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(qs=-1), dict(ks=1 << 40),
                                dict(qos=1023), dict(kos=255), dict(hq=-1), dict(hkv=-1), dict(q=FAKE + 1), dict(qs=2048)])
def test_bad_rows(kw):
    b, keep = _batch([3], [4])
    st, msg = _qk(_norm(), _rope(), b, **kw)
    assert st == EINVAL and msg


def test_null_structs_and_lengths():
    b, keep = _batch([3], [4])
    assert _qk(None, _rope(), b)[0] == EINVAL and _qk(_norm(), None, b)[0] == EINVAL and _qk(_norm(), _rope(), None)[0] == EINVAL
    assert _append(_norm(), _rope(), b, None)[0] == EINVAL and _append(None, _rope(), b, _cache())[0] == EINVAL
    assert _append(_norm(), _rope(), b, _cache(), v=None)[0] == EINVAL
    assert _append(_norm(), _rope(), b, _cache(head_dim=64, dtype=2))[0] == ENOTSUP
    bad, keep2 = _batch([1000], [25])
    assert _append(_norm(), _rope(), bad, _cache(dtype=2))[0] == ERANGE


@pytest.mark.parametrize("call", [
    lambda c, b: _status("s2l_kv_append", byref(c), byref(b), FAKE, FAKE, None),
    lambda c, b: _status("s2l_kv_gather", byref(c), byref(b), 0, FAKE, FAKE, FAKE, None),
    lambda c, b: _status("s2l_kv_swap_out", byref(c), FAKE, 1, FAKE, FAKE, 4, None),
    lambda c, b: _status("s2l_chunk_prefill_attn_noalloc", byref(c), byref(b), FAKE, 4, 0.1, FAKE, None, None, None, None),
    lambda c, b: _read(c, b), lambda c, b: _append(_norm(), _rope(), b, c)])
def test_bad_mxfp4_caches(call):
    b, keep = _batch([3], [4])
    scaled, k_off, v_off = _cache(dtype=2, scales=True), _cache(dtype=2), _cache(dtype=2)
    k_off.k_pages, v_off.v_pages = FAKE + 8, FAKE + 4
    for c in (scaled, k_off, v_off, _cache(dtype=3)):
        st, msg = call(c, b)
        assert st == EINVAL and msg, msg
    for c in (_cache(dtype=2, head_dim=64), _cache(dtype=2, page_size=32)):
        assert call(c, b)[0] == ENOTSUP


@pytest.mark.parametrize("scale", [2.0 ** -121, 1e-45, 2.0 ** 121])
def test_softmax_scales_past_the_queries_terms(scale):
    b, keep = _batch([3], [4])
    for cols in (128, 256):
        c, info = _cache(dtype=2), _lib.s2l_plan_info(tile_cols=cols)
        st, msg = _status("s2l_chunk_prefill_attn", byref(c), byref(b), FAKE, 4, scale, FAKE, None, byref(info), FAKE, 1 << 20, None)
        assert st == ENOTSUP and "softmax_scale" in msg


def test_quantised_queries_need_e4m3_pages():
    b, keep = _batch([3], [4])
    c, info = _cache(dtype=2), _lib.s2l_plan_info(tile_cols=128)
    st, msg = _status("s2l_chunk_prefill_attn_q8", byref(c), byref(b), FAKE, 4, 0.1, FAKE, None, byref(info), FAKE, 1 << 20, None)
    assert st == ENOTSUP and "e4m3" in msg


@pytest.mark.parametrize("kw,status", [(dict(part=-1), EINVAL), (dict(part=3), EINVAL), (dict(cu=None), EINVAL), (dict(k=None), EINVAL),
                                       (dict(v=None), EINVAL), (dict(k=FAKE + 8), EINVAL), (dict(v=FAKE + 2), EINVAL), (dict(rows=-1), EINVAL)])
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_bad_reads(kw, status, dtype):
    b, keep = _batch([3], [4])
    st, msg = _read(_cache(dtype=dtype, scales=dtype == 1), b, **kw)
    assert st == status and msg


def test_reads_of_bad_batches():
    for P, C, status in (([-1], [4], EINVAL), ([0], [-1], EINVAL), ([1000], [25], ERANGE), ([0] * 65536, [0] * 65536, ENOTSUP)):
        b, keep = _batch(P, C)
        assert _read(_cache(dtype=2), b)[0] == status
    b, keep = _batch([1 << 28], [1], max_pages=1 << 25)
    assert _read(_cache(dtype=2), b)[0] == ENOTSUP
    b, keep = _batch([3], [4])
    assert _read(_cache(dtype=2, hkv=65536), b)[0] == ENOTSUP
    assert _read(None, b)[0] == EINVAL and _read(_cache(), None)[0] == EINVAL
    b.block_tables = None
    assert _read(_cache(), b)[0] == EINVAL


def test_the_package_s_pools():
    pool = torch.zeros((3, 2, s2l.MXFP4_RUN_BYTES), dtype=torch.uint8)
    cache = s2l.PagedKVCache(pool, pool.clone())
    c = cache.c()
    assert cache.mxfp4 and not cache.fp8 and (c.dtype, c.num_pages, c.num_kv_heads, c.head_dim, c.page_size) == (2, 3, 2, 128, 16)
    assert not c.k_scale and not s2l.PagedKVCache(*(torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16) for _ in "kv")).mxfp4
    for k, v, kw in ((torch.zeros((3, 2, 1024), dtype=torch.uint8),) * 2 + ({},), (pool, pool[:2], {}),
                     (pool, pool, dict(k_scale=torch.ones(2))), (pool, pool.view(torch.int8), {}),
                     (torch.zeros((3, 2, 2 * s2l.MXFP4_RUN_BYTES), dtype=torch.uint8)[..., ::2], pool, {})):
        with pytest.raises(ValueError):
            s2l.PagedKVCache(k, v, **kw)
    cache.v_pages = pool[:2]          # set later: found by the next call
    with pytest.raises(ValueError):
        cache.c()
    cache.k_pages = cache.v_pages = torch.zeros((3, 2, 16, 128), dtype=torch.uint8)
    with pytest.raises(ValueError):
        cache.c()


def test_the_package_s_norms():
    w = torch.ones(128)
    assert s2l.QKNorm(w, w).c(w.device).weight_dtype == 1 and s2l.QKNorm(None, w.bfloat16()).c(w.device).weight_dtype == 0
    none = s2l.QKNorm().c(w.device)
    assert not none.q_weight and not none.k_weight
    for q, k in ((w, w.bfloat16()), (w[:64], None), (None, w.half()), (torch.ones(256)[::2], None), (w.view(1, 128), None)):
        with pytest.raises(ValueError):
            s2l.QKNorm(q, k)
    with pytest.raises(ValueError, match="q_weight is on cpu"):
        s2l.QKNorm(w).c(torch.device("meta"))


def test_the_package_s_calls():
    batch = s2l.Batch([16], [4], np.zeros((1, 2), np.int32), device="cpu")
    pool = torch.zeros((2, 2, s2l.MXFP4_RUN_BYTES), dtype=torch.uint8)
    cache = s2l.PagedKVCache(pool, pool.clone())
    out = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    good = dict(cu=batch.cu_chunk, k=out, v=out.clone())
    for kw, word in ((dict(cu=batch.cu_chunk.long()), "cu_out"), (dict(cu=batch.cu_chunk[:0]), "cu_out"), (dict(k=out.float()), "k_out"),
                     (dict(v=out[:3]), "v_out"), (dict(k=out[:, :1].contiguous()), "k_out"), (dict(v=out[..., :64].contiguous()), "v_out"),
                     (dict(k=torch.zeros((4, 4, 128), dtype=torch.bfloat16)[:, ::2]), "k_out"),
                     (dict(k=out.to("meta")), "k_out is on meta"), (dict(cu=batch.cu_chunk.to("meta")), "cu_out is on meta")):
        a = {**good, **kw}
        with pytest.raises(ValueError, match=word):
            s2l.s2l_kv_read(cache, batch, 2, a["cu"], a["k"], a["v"], 0)
    away = s2l.PagedKVCache(pool, pool.to("meta"))
    with pytest.raises(ValueError, match="v_pages is on meta"):
        s2l.s2l_kv_read(away, batch, 2, good["cu"], good["k"], good["v"], 0)
    for norm in (None, 3, torch.ones(128)):
        with pytest.raises(ValueError, match="QKNorm"):
            s2l.s2l_norm_rope_qk(batch, norm, s2l.Rope(torch.ones(64)), out, out, stream=0)
        with pytest.raises(ValueError, match="QKNorm"):
            s2l.s2l_norm_rope_kv_append(cache, batch, norm, s2l.Rope(torch.ones(64)), None, None, out, out, stream=0)
