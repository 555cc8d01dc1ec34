"""GPU: normed rows of 7, 8 and 11 groups of eight heads, of which a lane takes four, two or one, give the same bits."""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from tests.gpu_util import DEV
from tests.test_gpu_norm_rope import caches, weights
from tests.test_gpu_rope import freqs, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("kind,hq,hkv", [(None, 48, 8), (None, 40, 24), (None, 80, 7), ("bf16", 40, 8), ("fp8", 40, 8), ("fp8", 70, 9),
                                         ("mxfp4", 40, 8), ("mxfp4", 70, 9), ("mxfp4", 64, 8)])
def test_many_rows_give_the_bits_of_few(kind, hq, hkv, adjacent):
    """A large batch against batches of 40 rows, where a lane takes one head."""
    gen = torch.Generator(device=DEV).manual_seed(hq)
    T = 40 * 26                                    # 26 * 40 rows of 6 groups and more are past 6144 waves
    assert T * -(-(hq + hkv * (1 if kind is None else 2)) // 8) > 6144
    norm = s2l.QKNorm(*(weights((torch.bfloat16, 0.0), gen)[0] for _ in range(2)))
    rope = s2l.Rope(torch.from_numpy(freqs(48)).to(DEV), adjacent=adjacent)
    qkv = torch.randn((T, hq + 2 * hkv, 128), generator=gen, device=DEV).to(torch.bfloat16)
    pages = -(-T // 16)
    tables = np.random.default_rng(hq).permutation(pages).astype(np.int32)[None]
    outs = []
    for cache, parts in zip(caches(kind or "bf16", pages, hkv, gen), ([(0, T)], [(a, 40) for a in range(0, T, 40)])):
        q, k = (torch.zeros((T, n, 128), dtype=torch.bfloat16, device=DEV) for n in (hq, hkv))
        for a, n in parts:
            batch, row = s2l.Batch([a], [n], tables), qkv[a:a + n]
            if kind is None:
                s2l.s2l_norm_rope_qk(batch, norm, rope, row[:, :hq], q[a:a + n], row[:, hq:hq + hkv], k[a:a + n])
            else:
                s2l.s2l_norm_rope_kv_append(cache, batch, norm, rope, row[:, :hq], q[a:a + n], row[:, hq:hq + hkv], row[:, hq + hkv:])
        torch.cuda.synchronize()
        outs.append((q, k, cache.k_pages, cache.v_pages))
    assert all(same(x, y) for x, y in zip(*outs))
