"""GPU: attention over MXFP4 pages takes bf16 queries as they are, in every layout, however their sizes differ."""
import numpy as np
import pytest
import torch

import workloads
from oracle.paged_kv import bf16_bits_to_f32
from tests.gpu_util import assert_attention_close, to_bf16
from tests.mxfp4_util import MxSetup, mx_case, quantised_bits
from tests.test_gpu_mxfp4_attention import LAYOUTS, opts_of

pytestmark = pytest.mark.gpu

LARGE = [5, 37, 69]     # one dim of each of the first three blocks of 32


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("ratio", [30.0, 100.0, 2000.0, 2.0 ** 40])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_small_queries_beside_large_ones(layout, ratio, split):
    """Three dims hold queries `ratio` times the others', and keys of zero: their products are zeros, so the result
    is the one without them, bit for bit, and as near to the definition as with every other page type."""
    hq, hkv = 8, 2
    tq = layout[0] // (hq // hkv)
    case = mx_case("large", [400, 0], [2, tq + 1], hq, hkv, seed=80)
    q, k = bf16_bits_to_f32(case.q_bits), bf16_bits_to_f32(case.k_full_bits)
    k[:, :, LARGE] = 0
    q[:, :, LARGE] = 0
    plain = workloads.bf16_bits(q)
    q[:, :, LARGE] = (ratio * np.random.default_rng(80).choice([-1.0, 1.0], q[:, :, LARGE].shape)).astype(np.float32)
    case.k_full_bits, case.q_bits = quantised_bits(workloads.bf16_bits(k)), workloads.bf16_bits(q)
    s = MxSetup(case)
    s.append()
    out, lse = s.attention(opts_of(layout, split))
    assert s.plan.tile_cols == layout[0]
    assert_attention_close(case, out, lse, s.oracle(), what=f"{layout} {ratio}")
    s.q = to_bf16(plain)
    without, without_lse = s.attention(opts_of(layout, split))
    assert torch.equal(out.view(torch.int16), without.view(torch.int16)) and torch.equal(lse, without_lse)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_queries_of_many_binades_in_a_block(layout):
    """Queries of 25 binades side by side in each block."""
    case = mx_case("binades", [300], [5], 4, 2, seed=81)
    rng = np.random.default_rng(81)
    q = rng.standard_normal((5, 4, 128)) * 2.0 ** rng.integers(-22, 3, (5, 4, 128))
    case.q_bits = workloads.bf16_bits(q.astype(np.float32))
    s = MxSetup(case)
    s.append()
    out, lse = s.attention(opts_of(layout))
    assert_attention_close(case, out, lse, s.oracle(), what=f"{layout}")
