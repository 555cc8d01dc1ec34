"""MXFP4 pools set on a cache after it was made are looked at by the next call, on the native path too (CPU: every call is
refused before the library is asked)."""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from paper_2604_16395_amd import _lib

RUN = s2l.MXFP4_RUN_BYTES


def pool():
    return torch.zeros((3, 2, RUN), dtype=torch.uint8)


WRONG = [
    dict(v_pages=pool()[:2]), dict(v_pages=pool()[:, :1].contiguous()), dict(v_pages=torch.zeros((1, 1, 8))),
    dict(v_pages=pool().view(torch.int8)), dict(k_pages=pool().view(torch.int8)), dict(k_pages=torch.zeros((3, 2, RUN), dtype=torch.bfloat16)),
    dict(v_pages=torch.zeros((3, 2, 2 * RUN), dtype=torch.uint8)[..., ::2]), dict(k_pages=torch.zeros((6, 2, RUN), dtype=torch.uint8)[::2]),
    dict(k_pages=pool()[:2]), dict(k_pages=torch.zeros((3, 2, RUN + 16), dtype=torch.uint8)),
    dict(k_pages=torch.zeros((3, 2, 16, 128), dtype=torch.uint8), v_pages=torch.zeros((3, 2, 16, 128), dtype=torch.uint8)),
]


@pytest.mark.parametrize("wrong", WRONG)
def test_pools_set_later(wrong):
    cache = s2l.PagedKVCache(pool(), pool())
    for name, t in wrong.items():
        setattr(cache, name, t)
    batch = s2l.Batch([16], [4], np.zeros((1, 2), np.int32), device="cpu")
    row, q = (torch.zeros((4, h, 128), dtype=torch.bfloat16) for h in (2, 8))
    info = s2l.s2l_plan_host([16], [4], 8, 2)[0]
    ws = torch.zeros(info.workspace_bytes, dtype=torch.uint8)
    counts = torch.zeros(2, dtype=torch.int32)
    assert s2l._load_native() is not _lib._NoBinding
    for call in (lambda: s2l.s2l_kv_append(cache, batch, row, row, 0),
                 lambda: s2l.s2l_chunk_prefill_attn(cache, batch, q, 8, 0.1, q, None, info, ws, 0),
                 lambda: s2l.s2l_attn_main(cache, batch, q, 8, 0.1, q, None, info, ws, 0),
                 lambda: s2l.s2l_append_chunk_prefill_attn(cache, batch, row, row, q, 8, 0.1, q, None, info, ws, 0),
                 lambda: s2l.s2l_chunk_prefill_attn_noalloc(cache, batch, q, 8, 0.1, q, None, None, 0),
                 lambda: s2l.s2l_kv_gather(cache, batch, 1, counts, row, row, 0),
                 lambda: s2l.s2l_kv_read(cache, batch, s2l.S2L_READ_CHUNK, batch.cu_chunk, row, row.clone(), 0),
                 lambda: s2l.s2l_check_tables(cache, batch, counts, 0)):
        with pytest.raises(ValueError):
            call()
