"""GPU: norms of queries and keys with their rotation, and the append of normed rows, against float64.

With x the head, r = 1 / sqrt(mean x^2 + eps), n_d = x_d r (w_d + o): the sum of 128 squares in fp32 is off by at
most (16 + 3 + 1) roundings of 2^-24 (16 fused steps and three sums a lane, the mean and eps in one more; all
terms positive), half of it in the root, which has an error of its own of 1 ulp (2^-23), and two products and
the weight's sum add 3 roundings: |err n| <= (10 + 2 + 3) 2^-24 |n| < 2^-20 |n|.  The rotation acts on the normed
pair as on any other: |err| <= 2^-8 |y| + (2^-18 + 2^-20) (|a| + |b|) scale, and 2^-20 |n| where dims pass through.
"""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from oracle import mxfp4
from oracle.paged_kv import bf16_bits_to_f32
from oracle.qk_norm import norm_heads
from oracle.rotary import positions_of, rotate
from tests.gpu_util import DEV, bf16_to_f64, from_bf16
from tests.test_gpu_rope import CASES, freqs, positions_for, rows, same

pytestmark = pytest.mark.gpu


def weights(kind, gen):
    if kind is None:
        return None, 0.0
    dtype, offset = kind
    return (1 - offset + 0.5 * torch.randn(128, generator=gen, device=DEV)).to(dtype), offset


def check(y, x, w, eps, offset, pos, inv, axes, adjacent, scale=1.0):
    n = norm_heads(bf16_to_f64(x), None if w is None else w.double().cpu().numpy(), np.float32(eps), offset)
    ref, reach = rotate(n, pos, inv, axes, adjacent, scale)
    err = np.abs(bf16_to_f64(y) - ref)
    through = np.where(reach > 0, 0.0, np.abs(n))
    bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -18 + 2.0 ** -20) * reach + 2.0 ** -19 * through + 1e-37
    worst = np.unravel_index(np.argmax(err - bound), err.shape)
    assert np.all(err <= bound), (worst, err[worst], bound[worst])


WEIGHTS = [None, (torch.bfloat16, 0.0), (torch.float32, 0.0), (torch.bfloat16, 1.0), (torch.float32, 1.0)]


@pytest.mark.parametrize("kind", WEIGHTS)
@pytest.mark.parametrize("case", CASES)
def test_normed_rotation_equals_the_definition(case, kind):
    P, C, hq, hkv, rot, sections, cyclic, adjacent = case
    gen = torch.Generator(device=DEV).manual_seed(1)
    T, inv = sum(C), freqs(rot // 2)
    axes = [0] * (rot // 2) if sections is None else s2l.rope_pair_axes(sections, cyclic)
    dev_pos, pos = positions_for(case, gen)
    batch = s2l.Batch(P, C, np.zeros((len(P), 1), np.int32))
    rope = s2l.Rope(torch.from_numpy(inv).to(DEV), dev_pos, axes, adjacent, 1.25)
    (qw, offset), (kw, _) = weights(kind, gen), weights(kind, gen)
    norm = s2l.QKNorm(qw, kw, 1e-5, offset)
    qkv = rows(gen, T, hq + 2 * hkv, pad=2)
    qkv *= torch.exp(2 * torch.randn((T + 2, hq + 2 * hkv, 1), generator=gen, device=DEV)).to(torch.bfloat16)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    before = qkv.clone()
    q_out, k_out = torch.full((T + 2, hq, 128), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((T + 2, hkv + 1, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    s2l.s2l_norm_rope_qk(batch, norm, rope, q, q_out, k, k_out[:, :hkv])
    torch.cuda.synchronize()
    check(q_out[:T], q[:T], qw, 1e-5, offset, pos, inv, axes, adjacent, 1.25)
    check(k_out[:T, :hkv], k[:T], kw, 1e-5, offset, pos, inv, axes, adjacent, 1.25)
    assert bool((q_out[T:] == 7).all()) and bool((k_out[T:] == 7).all()) and bool((k_out[:, hkv:] == 7).all())
    assert same(qkv, before)
    only = torch.empty_like(q_out[:T])      # without keys, and in place
    s2l.s2l_norm_rope_qk(batch, norm, rope, q, only)
    s2l.s2l_norm_rope_qk(batch, norm, rope, q, q, k, k)
    torch.cuda.synchronize()
    assert same(only, q_out[:T]) and same(q[:T], q_out[:T]) and same(k[:T], k_out[:T, :hkv])
    assert same(qkv[:, hq + hkv:], before[:, hq + hkv:]) and same(qkv[T:], before[T:])


def caches(kind, pages, hkv, gen):
    if kind == "mxfp4":
        pools = [torch.randint(0, 256, (pages, hkv, mxfp4.RUN), dtype=torch.uint8, generator=gen, device=DEV) for _ in range(2)]
        return [s2l.PagedKVCache(*(p.clone() for p in pools)) for _ in range(2)]
    if kind == "fp8":
        pools = [torch.randint(0, 256, (pages, hkv, 16, 128), dtype=torch.uint8, generator=gen, device=DEV) for _ in range(2)]
        scales = [0.01 + torch.rand(hkv, generator=gen, device=DEV) for _ in range(2)]
        return [s2l.PagedKVCache(*(p.clone() for p in pools), *scales) for _ in range(2)]
    pools = [torch.randn((pages, hkv, 16, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2)]
    return [s2l.PagedKVCache(*(p.clone() for p in pools)) for _ in range(2)]


@pytest.mark.parametrize("kind", ["bf16", "fp8", "mxfp4"])
@pytest.mark.parametrize("rot,adjacent", [(128, False), (96, False), (16, False), (64, True)])
def test_normed_append_is_norm_and_rotation_then_append(kind, rot, adjacent):
    """Pages and q_out of the one call bit for bit those of the two, with one head a lane and with two, without
    queries, and with groups of eight heads that hold queries, keys and values."""
    gen = torch.Generator(device=DEV).manual_seed(rot)
    rope = s2l.Rope(torch.from_numpy(freqs(rot // 2)).to(DEV), adjacent=adjacent)
    norm = s2l.QKNorm(*(weights((torch.bfloat16, 0.0), gen)[0] for _ in range(2)), 1e-6)
    for P, C, hq, hkv in (([2047], [1], 8, 2), ([5, 0, 30], [33, 0, 21], 0, 5), ([3], [20], 5, 3), ([7, 100], [700, 1200], 32, 8)):
        need = [-(-(p + c) // 16) for p, c in zip(P, C)]
        tables = np.zeros((len(P), max(need)), np.int32)
        for r, n in enumerate(need):
            tables[r, :n] = sum(need[:r]) + np.arange(n)
        one, two = caches(kind, sum(need), hkv, gen)
        batch, T = s2l.Batch(P, C, tables), sum(C)
        qkv = torch.randn((T, hq + 2 * hkv, 128), generator=gen, device=DEV).to(torch.bfloat16)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        q1, q2, k2 = (torch.zeros((T, n, 128), dtype=torch.bfloat16, device=DEV) for n in (hq, hq, hkv))
        s2l.s2l_norm_rope_kv_append(one, batch, norm, rope, q if hq else None, q1 if hq else None, k, v)
        s2l.s2l_norm_rope_qk(batch, norm, rope, q, q2, k, k2)
        s2l.s2l_kv_append(two, batch, k2, v.contiguous())
        torch.cuda.synchronize()
        assert same(q1, q2) and same(one.k_pages, two.k_pages) and same(one.v_pages, two.v_pages), (P, C)


@pytest.mark.parametrize("hq,hkv", [(4, 2), (12, 2), (20, 7), (30, 1), (32, 8), (64, 8)])
@pytest.mark.parametrize("kind", [None, "bf16", "mxfp4"])
def test_many_rows_give_the_bits_of_few(hq, hkv, kind):
    """One to four heads a lane, with a wave's heads queries, keys and values in any mix: the rows of a large batch have
    the bits that they have in batches of 40 rows, where a lane takes one head."""
    gen = torch.Generator(device=DEV).manual_seed(hq)
    heads = hq + hkv * (1 if kind is None else 2)
    T = 40 * (6144 // (-(-heads // 8) * 40) + 2)
    norm = s2l.QKNorm(*(weights((torch.float32, 0.0), gen)[0] for _ in range(2)))
    rope = s2l.Rope(torch.from_numpy(freqs(48)).to(DEV))
    qkv = torch.randn((T, hq + 2 * hkv, 128), generator=gen, device=DEV).to(torch.bfloat16)
    pages = -(-T // 16)
    tables = np.random.default_rng(hq).permutation(pages).astype(np.int32)[None]
    many, few = caches(kind or "bf16", pages, hkv, gen)
    outs = []
    for cache, parts in ((many, [(0, T)]), (few, [(a, 40) for a in range(0, T, 40)])):
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


def test_weights_and_rows_at_odd_addresses():
    gen = torch.Generator(device=DEV).manual_seed(3)
    T, hq, inv = 37, 3, freqs(64)
    batch, rope = s2l.Batch([10], [T], np.zeros((1, 1), np.int32)), s2l.Rope(torch.from_numpy(inv).to(DEV))
    flat = torch.randn(1 + T * (hq * 128 + 5), generator=gen, device=DEV).to(torch.bfloat16)
    q = flat[1:].view(T, -1)[:, :hq * 128].unflatten(1, (hq, 128))
    pos = positions_of([10], [T])[None]
    for dtype in (torch.bfloat16, torch.float32):
        w = torch.randn(131, generator=gen, device=DEV).to(dtype)[3:]
        room = torch.zeros(3 + T * (hq * 128 + 1), dtype=torch.bfloat16, device=DEV)
        out = room[3:].view(T, -1)[:, :hq * 128].unflatten(1, (hq, 128))
        s2l.s2l_norm_rope_qk(batch, s2l.QKNorm(w, None, 1e-6), rope, q, out)
        torch.cuda.synchronize()
        check(out, q, w, 1e-6, 0.0, pos, inv, [0] * 64, False)
        assert not room[:3].any() and not room[3:].view(T, -1)[:, hq * 128:].any()


def test_heads_of_zeros_of_far_sizes_and_not_finite():
    """A head of zeros stays zero, sizes from 2^-60 to 2^55 are normed as their definition, and a NaN or an infinity
    stays within its head."""
    T, inv = 6, freqs(64)
    gen = torch.Generator(device=DEV).manual_seed(4)
    q = rows(gen, T, 5)
    q[0], q[1], q[2] = 0, q[1] * 2.0 ** 55, q[2] * 2.0 ** -60
    clean = q.clone()
    q[4, 1, 7], q[5, 3, 100] = float("nan"), float("inf")
    batch, rope = s2l.Batch([9], [T], np.zeros((1, 1), np.int32)), s2l.Rope(torch.from_numpy(inv).to(DEV))
    out, ref = torch.empty_like(q), torch.empty_like(q)
    norm = s2l.QKNorm(eps=1e-30)
    s2l.s2l_norm_rope_qk(batch, norm, rope, q, out)
    s2l.s2l_norm_rope_qk(batch, norm, rope, clean, ref)
    torch.cuda.synchronize()
    check(ref, clean, None, 1e-30, 0.0, positions_of([9], [T])[None], inv, [0] * 64, False)
    assert torch.isnan(out[4, 1]).all() and torch.isnan(out[5, 3, [100, 36]]).all()
    out[4, 1], out[5, 3] = ref[4, 1], ref[5, 3]
    assert same(out, ref)


def test_values_are_not_normed():
    gen = torch.Generator(device=DEV).manual_seed(5)
    cache = caches("bf16", 2, 3, gen)[0]
    batch, rope = s2l.Batch([0], [20], np.array([[1, 0]], np.int32)), s2l.Rope(torch.from_numpy(freqs(64)).to(DEV))
    kv = 9 * torch.randn((20, 6, 128), generator=gen, device=DEV).to(torch.bfloat16)
    s2l.s2l_norm_rope_kv_append(cache, batch, s2l.QKNorm(), rope, None, None, kv[:, :3], kv[:, 3:])
    torch.cuda.synchronize()
    got = torch.cat([cache.v_pages[1].transpose(0, 1), cache.v_pages[0].transpose(0, 1)])[:20]
    assert np.array_equal(from_bf16(got), from_bf16(kv[:, 3:]))


def test_normed_keys_in_mxfp4_pages_are_quantised_normed_keys():
    """The pages' values against the definition: the quantised form of what the normed rotation gives."""
    gen = torch.Generator(device=DEV).manual_seed(6)
    cache = caches("mxfp4", 2, 2, gen)[0]
    batch, rope = s2l.Batch([0], [20], np.array([[1, 0]], np.int32)), s2l.Rope(torch.from_numpy(freqs(64)).to(DEV))
    norm = s2l.QKNorm(None, weights((torch.float32, 0.0), gen)[0])
    kv = torch.randn((20, 4, 128), generator=gen, device=DEV).to(torch.bfloat16)
    k = torch.empty((20, 2, 128), dtype=torch.bfloat16, device=DEV)
    s2l.s2l_norm_rope_kv_append(cache, batch, norm, rope, None, None, kv[:, :2], kv[:, 2:])
    s2l.s2l_norm_rope_qk(batch, s2l.QKNorm(norm.k_weight, None), rope, kv[:, :2], k)
    torch.cuda.synchronize()
    page, slot = [1] * 16 + [0] * 4, list(range(16)) + list(range(4))
    for pool, x in ((cache.k_pages, k), (cache.v_pages, kv[:, 2:])):
        want = mxfp4.dequantise(*mxfp4.quantise(bf16_bits_to_f32(from_bf16(x)).astype(np.float64)))
        assert np.array_equal(mxfp4.load(pool.cpu().numpy(), page, slot)[1], want)
