"""Attention without a workspace refuses a softmax scale out of range over MXFP4 pages before its plan is enqueued (CPU: an
enqueued plan would have failed for want of a device)."""
import ctypes

import pytest

from paper_2604_16395_amd import _lib
from tests.test_abi_cpu import FAKE, _batch, _cache, _status


@pytest.mark.parametrize("scale", [2.0 ** -121, 1e-45, 2.0 ** 121])
@pytest.mark.parametrize("cols", [128, 256])
def test_scales_out_of_range(scale, cols):
    b, keep = _batch([3], [40])
    c, opts = _cache(dtype=2), _lib.s2l_plan_opts(target_items=64, tile_cols=cols)
    st, msg = _status("s2l_chunk_prefill_attn_noalloc", ctypes.byref(c), ctypes.byref(b), FAKE, 4, scale, FAKE, None, ctypes.byref(opts), None, None)
    assert st == _lib.S2L_ENOTSUP and "softmax_scale" in msg
