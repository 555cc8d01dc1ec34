"""GPU: the rotation and the rotating append over enough rows for two heads a lane (more than 6144 waves of 8 heads of a row),
where a group of 16 heads can hold queries, keys and values at once; bounds as in test_gpu_rope."""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from oracle.rotary import positions_of
from tests.gpu_util import DEV
from tests.test_gpu_rope import check, freqs, pools, rows, same

pytestmark = pytest.mark.gpu
EVERY = 89      # of the rows, against float64


def case(C, P, hq, hkv, rot, sections, adjacent, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T, inv = sum(C), freqs(rot // 2)
    axes = [0] * (rot // 2) if sections is None else s2l.rope_pair_axes(sections, True)
    dev_pos = None if sections is None else torch.randint(-9, 70000, (len(sections), T), generator=gen, device=DEV, dtype=torch.int32)
    pos = positions_of(P, C)[None] if sections is None else dev_pos.cpu().numpy()
    rope = s2l.Rope(torch.from_numpy(inv).to(DEV), dev_pos, axes, adjacent)
    qkv = rows(gen, T, hq + 2 * hkv)
    some = slice(0, T, EVERY)
    return rope, qkv, lambda y, x: check(y[some], x[some], pos[:, some], inv, axes, adjacent)


# the last: one head a lane for s2l_rope_qk (3000 rows of two groups of 8 heads), two for the append (of three)
SHAPES = [([8000, 3, 997], 17, 2), ([1, 8999], 9, 9), ([9000], 8, 1), ([2900, 100], 8, 8)]


@pytest.mark.parametrize("rot,sections,adjacent", [(128, None, False), (96, None, True), (128, (24, 20, 20), False), (64, (16, 16), True)])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("C,hq,hkv", SHAPES)
def test_wide_append(C, hq, hkv, fp8, rot, sections, adjacent):
    """Pages and queries bit for bit those of s2l_rope_qk and s2l_kv_append."""
    print(f"[rope wide] {C} {hq}/{hkv} fp8={fp8} {rot} {sections} {adjacent}", flush=True)
    P = [37 * (r + 1) for r in range(len(C))]
    rope, qkv, against_float64 = case(C, P, hq, hkv, rot, sections, adjacent, seed=70)
    need = [(p + c + 15) // 16 for p, c in zip(P, C)]
    order = np.random.default_rng(70).permutation(sum(need) + 2)
    tables = np.full((len(P), max(need)), -1, np.int32)
    for r, n in enumerate(need):
        tables[r, :n] = order[sum(need[:r]):sum(need[:r]) + n]
    kp, vp, ks, vs = pools(sum(need) + 2, hkv, fp8, torch.Generator(device=DEV).manual_seed(71))
    batch = s2l.Batch(P, C, tables)
    cache, ref = s2l.PagedKVCache(kp.clone(), vp.clone(), ks, vs), s2l.PagedKVCache(kp, vp, ks, vs)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    q_out, q_ref, k_ref = (torch.full(t.shape, 7.0, dtype=t.dtype, device=DEV) for t in (q, q, k))
    s2l.s2l_rope_kv_append(cache, batch, rope, q, q_out, k, v)
    s2l.s2l_rope_qk(batch, rope, q, q_ref, k, k_ref)
    s2l.s2l_kv_append(ref, batch, k_ref, v.contiguous())
    torch.cuda.synchronize()
    assert same(q_out, q_ref) and same(cache.k_pages, ref.k_pages) and same(cache.v_pages, ref.v_pages)
    against_float64(q_out, q)
    against_float64(k_ref, k)
    # keys and values alone, queries alone
    alone, q_alone = s2l.PagedKVCache(cache.k_pages.clone(), cache.v_pages.clone(), ks, vs), torch.zeros_like(q_out)
    s2l.s2l_rope_kv_append(alone, batch, rope, None, None, k, v)
    s2l.s2l_rope_qk(batch, rope, q, q_alone)
    torch.cuda.synchronize()
    assert same(alone.k_pages, ref.k_pages) and same(alone.v_pages, ref.v_pages) and same(q_alone, q_ref)


@pytest.mark.parametrize("hq,hkv", [(17, 2), (9, 9), (1, 33)])
def test_wide_adjacent_pairs(hq, hkv):
    C, P = [8000, 1000], [5, 1000]
    rope, qkv, against_float64 = case(C, P, hq, hkv, 96, None, True, seed=72)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    q_out, k_out = torch.zeros(q.shape, dtype=q.dtype, device=DEV), torch.zeros(k.shape, dtype=k.dtype, device=DEV)
    s2l.s2l_rope_qk(s2l.Batch(P, C, np.zeros((2, 1), np.int32)), rope, q, q_out, k, k_out)
    torch.cuda.synchronize()
    against_float64(q_out, q)
    against_float64(k_out, k)
