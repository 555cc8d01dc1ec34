"""GPU: the norms at the smallest eps that they take, 2^-126, against float64 with the bound of test_gpu_norm_rope."""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from oracle.rotary import positions_of
from tests.gpu_util import DEV
from tests.test_gpu_norm_rope import check
from tests.test_gpu_rope import freqs, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [2.0 ** -126, 3e-38])
def test_smallest_eps(eps):
    """Heads of zeros stay zero; sizes from 2^-80, whose squares vanish beside eps as in float64, to 2^20."""
    T, inv = 6, freqs(64)
    q = rows(torch.Generator(device=DEV).manual_seed(6), T, 5)
    for i, size in enumerate((0.0, 2.0 ** -80, 2.0 ** -64, 2.0 ** -60, 1.0, 2.0 ** 20)):
        q[i] *= size
    batch, rope = s2l.Batch([9], [T], np.zeros((1, 1), np.int32)), s2l.Rope(torch.from_numpy(inv).to(DEV))
    out = torch.empty_like(q)
    s2l.s2l_norm_rope_qk(batch, s2l.QKNorm(eps=eps), rope, q, out)
    torch.cuda.synchronize()
    assert not out[0].any()
    check(out, q, None, eps, 0.0, positions_of([9], [T])[None], inv, [0] * 64, False)
