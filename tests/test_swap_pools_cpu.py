"""Host pools of another page size than the cache's are refused: copied by the cache's page size, they would be read and
written out of place and past their end (CPU: nothing is enqueued)."""
import pytest
import torch

import paper_2604_16395_amd as s2l


def cache(kind, hkv=2):
    if kind == "mxfp4":
        return s2l.PagedKVCache(*(torch.zeros((3, hkv, s2l.MXFP4_RUN_BYTES), dtype=torch.uint8) for _ in "kv"))
    pages = [torch.zeros((3, hkv, 16, 128), dtype=torch.uint8 if kind == "fp8" else torch.bfloat16) for _ in "kv"]
    return s2l.PagedKVCache(*pages, *([torch.ones(hkv)] * 2 if kind == "fp8" else []))


PAIRS = torch.zeros((1, 2), dtype=torch.int32)


@pytest.mark.parametrize("swap", [s2l.s2l_kv_swap_out, s2l.s2l_kv_swap_in])
@pytest.mark.parametrize("kind,shape", [
    ("mxfp4", (4, 2, 16, 128)), ("mxfp4", (4, 2, 1024)), ("mxfp4", (4, 1, s2l.MXFP4_RUN_BYTES)), ("mxfp4", (4,)), ("mxfp4", ()),
    ("fp8", (4, 2, s2l.MXFP4_RUN_BYTES)), ("fp8", (4, 1, 16, 128)), ("bf16", (4, 1, 16, 128)), ("bf16", (4, 2, 16, 64))])
def test_pools_of_other_pages(kind, shape, swap):
    c = cache(kind)
    pools = [torch.zeros(shape, dtype=c.k_pages.dtype) for _ in "kv"]
    with pytest.raises(ValueError, match="host pools must hold pages"):
        swap(c, PAIRS, *pools, 0)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "mxfp4"])
def test_pools_of_the_cache_s_pages(kind):
    """Whole pages in any shape are taken: what is refused next is `pairs`, which are not on a device."""
    c = cache(kind)
    for shape in ((4,) + tuple(c.k_pages.shape[1:]), (4, c.k_pages[0].numel())):
        pools = [torch.zeros(shape, dtype=c.k_pages.dtype) for _ in "kv"]
        with pytest.raises(ValueError, match="pairs must be a device"):
            s2l.s2l_kv_swap_out(c, PAIRS, *pools, 0)
