"""The smallest eps of the norms: below 2^-126 the hardware's root takes eps for zero, and a head of zeros would come out
as NaN."""

import pytest

from paper_2604_16395_amd import _lib
from tests.test_abi_cpu import _batch, _cache
from tests.test_mxfp4_norm_abi_cpu import _append, _norm, _qk
from tests.test_rope_linear_abi_cpu import _rope


@pytest.mark.parametrize("eps", [2.0 ** -127, 2.0 ** -149, 1e-40, 1.17e-38])
@pytest.mark.parametrize("dtype", [0, 2])
def test_denormal_eps_is_refused(eps, dtype):
    b, keep = _batch([3], [4])
    for st, msg in (_qk(_norm(eps=eps), _rope(), b), _append(_norm(eps=eps), _rope(), b, _cache(dtype=dtype))):
        assert st == _lib.S2L_EINVAL and "eps" in msg


def test_the_smallest_eps_is_taken():
    """What is refused next is the missing rotation."""
    b, keep = _batch([3], [4])
    st, msg = _qk(_norm(eps=2.0 ** -126), None, b)
    assert st == _lib.S2L_EINVAL and "rope" in msg
