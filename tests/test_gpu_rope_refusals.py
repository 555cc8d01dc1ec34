"""GPU: the rotating append refuses a cache that is not on the batch's device, marshalled natively or not; nothing is launched."""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from tests.gpu_util import DEV
from tests.test_gpu_rope import freqs, rows, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("away", ["k_pages", "v_pages", "k_scale", "v_scale"])
def test_a_cache_on_the_host_is_refused(monkeypatch, away, native):
    gen = torch.Generator(device=DEV).manual_seed(80)
    batch = s2l.Batch([3], [5], np.arange(4, dtype=np.int32)[None])
    rope = s2l.Rope(torch.from_numpy(freqs(64)).to(DEV))
    qkv = rows(gen, 5, 8)
    q, k, v, q_out = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], torch.full((5, 4, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    on = lambda n, t: t.cpu() if n == away else t  # noqa: E731
    cache = s2l.PagedKVCache(*(on(n, torch.zeros((4, 2, 16, 128), dtype=torch.uint8, device=DEV)) for n in ("k_pages", "v_pages")),
                             *(on(n, torch.ones(2, device=DEV)) for n in ("k_scale", "v_scale")))
    if not native:
        monkeypatch.setattr(s2l, "_native", s2l._lib._NoBinding)
    before = q_out.clone()
    with pytest.raises(ValueError, match=f"{away} is on cpu"):
        s2l.s2l_rope_kv_append(cache, batch, rope, q, q_out, k, v)
    torch.cuda.synchronize()
    assert same(q_out, before) and not any(bool(t.any()) for t in (cache.k_pages, cache.v_pages))
