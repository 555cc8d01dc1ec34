"""GPU: a module's parameters as the norms' weights give the bits of plain tensors."""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from tests.gpu_util import DEV
from tests.test_gpu_norm_rope import caches
from tests.test_gpu_rope import freqs, rows, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_parameters_give_the_bits_of_tensors(dtype, kind):
    gen = torch.Generator(device=DEV).manual_seed(7)
    w = [(1 + 0.3 * torch.randn(128, generator=gen, device=DEV)).to(dtype) for _ in "qk"]
    batch, rope = s2l.Batch([5], [20], np.array([[0, 1]], np.int32)), s2l.Rope(torch.from_numpy(freqs(64)).to(DEV))
    q, k, v = rows(gen, 20, 8), rows(gen, 20, 2), rows(gen, 20, 2)
    outs = []
    for norm, cache in zip((s2l.QKNorm(*w), s2l.QKNorm(*(torch.nn.Parameter(x) for x in w))), caches(kind, 2, 2, gen)):
        q1, q2, k2 = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k)
        s2l.s2l_norm_rope_kv_append(cache, batch, norm, rope, q, q1, k, v)
        s2l.s2l_norm_rope_qk(batch, norm, rope, q, q2, k, k2)
        torch.cuda.synchronize()
        outs.append((q1, q2, k2, cache.k_pages, cache.v_pages))
    assert all(same(a, b) for a, b in zip(*outs))
