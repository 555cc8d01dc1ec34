"""The MXFP4 gather writes words of four bytes: outputs off that are refused before anything is enqueued."""
import ctypes

import pytest

from paper_2604_16395_amd import _lib
from tests.test_abi_cpu import FAKE, _batch, _cache, _status


@pytest.mark.parametrize("k,v", [(FAKE + 1, FAKE), (FAKE, FAKE + 2), (FAKE + 3, FAKE + 3)])
@pytest.mark.parametrize("chunk", [0, 1])
def test_gather_outputs_off_four_bytes(k, v, chunk):
    b, keep = _batch([3], [4])
    st, msg = _status("s2l_kv_gather", ctypes.byref(_cache(dtype=2)), ctypes.byref(b), chunk, FAKE, k, v, None)
    assert st == _lib.S2L_EINVAL and "4 bytes" in msg
