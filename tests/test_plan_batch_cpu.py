"""A plan is for one batch's lengths: attention refuses it for a batch whose counts are the same and whose lengths are
not, before anything is enqueued (its items would read that batch's block tables and rows by another's lengths)."""
import ctypes

import pytest

from paper_2604_16395_amd import _lib
from tests.test_abi_cpu import FAKE, _batch, _cache, _plan, _status

byref = ctypes.byref
OTHERS = [  # prefixes and chunks of the plan, and of the batch: as many requests, tokens and items
    (([31], [40]), ([30], [40])),
    (([0], [1]), ([4095], [1])),
    (([100, 200], [3, 3]), ([200, 100], [3, 3])),
    (([100, 100], [3, 5]), ([100, 100], [5, 3])),
    (([64] * 40, [1] * 40), ([64] * 39 + [80], [1] * 40)),
]


def calls(cache, b, info, nbytes):
    attn = lambda name: _status(name, byref(cache), byref(b), FAKE, 8, 0.1, FAKE, None, byref(info), FAKE, nbytes, None)  # noqa: E731
    yield attn("s2l_attn_main")
    yield attn("s2l_chunk_prefill_attn")
    if info.tile_cols != 16 and cache.dtype == 1:
        yield attn("s2l_chunk_prefill_attn_q8")
    yield _status("s2l_append_chunk_prefill_attn", byref(cache), byref(b), FAKE, FAKE, FAKE, 8, 0.1, FAKE, None, byref(info), FAKE, nbytes,
                  byref(ctypes.c_int32()), None)


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("planned,given", OTHERS)
def test_a_plan_of_another_batch_s_lengths(planned, given, dtype):
    b, keep = _batch(*given, max_pages=512)
    cache = _cache(dtype=dtype, scales=dtype == 1)
    info = _plan(*planned, 8, 2)
    for st, msg in calls(cache, b, info, 1 << 40):
        assert st == _lib.S2L_EINVAL and "another batch" in msg, msg
    own = _plan(*given, 8, 2)     # the batch's own plan is taken as far as its workspace
    for st, msg in calls(cache, b, own, own.workspace_bytes - 1):
        assert st == _lib.S2L_EWORKSPACE, msg
    assert (own.num_reqs, own.total_tokens) == (info.num_reqs, info.total_tokens)
