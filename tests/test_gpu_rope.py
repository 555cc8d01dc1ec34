"""GPU: rotary positions (one axis and several) and the append that rotates, against float64.

A rotated value is rounded once to bf16 (half a step, 2^-8 of it) after fp32 arithmetic on a sine and a
cosine that are off by at most 2^-18 (angles are exact up to 2^-26 of a turn, the hardware's functions
and three fp32 roundings of 2^-24 come on top): |err| <= 2^-8 |y| + 2^-18 (|a| + |b|) scale.
"""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from oracle.paged_kv import bf16_bits_to_f32
from oracle.rotary import positions_of, rotate
from tests.gpu_util import DEV, bf16_to_f64, from_bf16

pytestmark = pytest.mark.gpu


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def freqs(pairs, base=10000.0):
    return (base ** -(np.arange(pairs) / pairs)).astype(np.float32)


def rows(gen, T, heads, pad=0):
    return torch.randn((T + pad, heads, 128), generator=gen, device=DEV).to(torch.bfloat16)


def check(y, x, pos, inv, axes, adjacent, scale=1.0):
    ref, reach = rotate(bf16_to_f64(x), pos, inv, axes, adjacent, scale)
    err = np.abs(bf16_to_f64(y) - ref)
    bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * reach
    worst = np.unravel_index(np.argmax(err - bound), err.shape)
    assert np.all(err <= bound), (worst, err[worst], bound[worst])
    rot = 2 * len(inv)
    assert np.array_equal(from_bf16(y)[..., rot:], from_bf16(x)[..., rot:])


CASES = [  # prefixes, chunks, hq, hkv, rotated dims, sections, cyclic, adjacent
    ([2047], [1], 32, 8, 128, None, False, False),
    ([0, 5, 100], [1, 3, 2], 8, 1, 64, None, False, False),
    ([3, 0, 0, 77], [0, 130, 1, 0], 4, 4, 96, None, False, True),
    ([500], [67], 5, 5, 128, (16, 24, 24), False, False),
    ([0, 9], [33, 40], 7, 1, 128, (24, 20, 20), True, False),
    ([0, 9], [33, 40], 3, 3, 32, (8, 8), False, True),
    ([1], [19], 64, 8, 16, (2, 2, 2, 2), True, False),
]


def positions_for(case, gen):
    P, C, sections = case[0], case[1], case[5]
    T = sum(C)
    if sections is None:
        return None, positions_of(P, C)[None]
    pos = torch.randint(-100, 5000, (len(sections), T + 3), generator=gen, device=DEV, dtype=torch.int32)
    return pos[:, :T], pos[:, :T].cpu().numpy()    # axes further apart than the rows


@pytest.mark.parametrize("case", CASES)
def test_rotation_equals_the_definition(case):
    P, C, hq, hkv, rot, sections, cyclic, adjacent = case
    print(f"[rope] {case}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(1)
    T, inv = sum(C), freqs(rot // 2)
    axes = [0] * (rot // 2) if sections is None else s2l.rope_pair_axes(sections, cyclic)
    dev_pos, pos = positions_for(case, gen)
    batch = s2l.Batch(P, C, np.zeros((len(P), 1), np.int32))
    rope = s2l.Rope(torch.from_numpy(inv).to(DEV), dev_pos, axes, adjacent)
    qkv = rows(gen, T, hq + 2 * hkv, pad=2)        # a projected row: queries and keys are views of it
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    before = qkv.clone()
    q_out, k_out = torch.full((T + 2, hq, 128), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((T + 2, hkv + 1, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    s2l.s2l_rope_qk(batch, rope, q, q_out, k, k_out[:, :hkv])
    torch.cuda.synchronize()
    check(q_out[:T], q[:T], pos, inv, axes, adjacent)
    check(k_out[:T, :hkv], k[:T], pos, inv, axes, adjacent)
    assert bool((q_out[T:] == 7).all()) and bool((k_out[T:] == 7).all()) and bool((k_out[:, hkv:] == 7).all())
    assert same(qkv, before)
    # without keys, and in place within the projected row
    only = torch.empty_like(q_out[:T])
    s2l.s2l_rope_qk(batch, rope, q, only)
    s2l.s2l_rope_qk(batch, rope, q, q, k, k)
    torch.cuda.synchronize()
    assert same(only, q_out[:T]) and same(q[:T], q_out[:T]) and same(k[:T], k_out[:T, :hkv])
    assert same(qkv[:, hq + hkv:], before[:, hq + hkv:]) and same(qkv[T:], before[T:])


def test_rows_at_odd_addresses_and_scaled():
    gen = torch.Generator(device=DEV).manual_seed(2)
    T, hq = 37, 3
    inv = freqs(64)
    flat = torch.randn(1 + T * (hq * 128 + 5), generator=gen, device=DEV).to(torch.bfloat16)
    q = flat[1:].view(T, -1)[:, :hq * 128].unflatten(1, (hq, 128))
    room = torch.zeros(3 + T * (hq * 128 + 1), dtype=torch.bfloat16, device=DEV)
    out = room[3:].view(T, -1)[:, :hq * 128].unflatten(1, (hq, 128))
    batch = s2l.Batch([10], [T], np.zeros((1, 1), np.int32))
    rope = s2l.Rope(torch.from_numpy(inv).to(DEV), scale=1.37)
    s2l.s2l_rope_qk(batch, rope, q, out)
    torch.cuda.synchronize()
    check(out, q, positions_of([10], [T])[None], inv, [0] * 64, False, float(np.float32(1.37)))
    assert int((room[:3] != 0).sum()) == 0 and int((room[3:].view(T, -1)[:, hq * 128:] != 0).sum()) == 0


@pytest.mark.parametrize("num_reqs", [64, 65, 700, 5000])
def test_rows_find_their_request(num_reqs):
    """Requests with and without rows, more than the search looks at in one and in two steps."""
    rng = np.random.default_rng(3)
    C = rng.integers(0, 3, num_reqs)
    C[0] = C[-1] = 0
    P = rng.integers(0, 1 << 20, num_reqs)
    T, inv = int(C.sum()), freqs(8)
    q = rows(torch.Generator(device=DEV).manual_seed(3), T, 1)
    out = torch.empty_like(q)
    s2l.s2l_rope_qk(s2l.Batch(P, C, np.zeros((num_reqs, 1), np.int32)), s2l.Rope(torch.from_numpy(inv).to(DEV)), q, out)
    torch.cuda.synchronize()
    check(out, q, positions_of(P, C)[None], inv, [0] * 8, False)


def test_far_positions_lose_nothing():
    P, C = [(1 << 30) - 40, 123_456_789, 1_000_003], [40, 17, 5]
    inv = np.concatenate([np.float32([1.0, 0.9999, 3.0, 0.5]), freqs(60)])
    q = rows(torch.Generator(device=DEV).manual_seed(4), sum(C), 2)
    out = torch.empty_like(q)
    s2l.s2l_rope_qk(s2l.Batch(P, C, np.zeros((3, 1), np.int32)), s2l.Rope(torch.from_numpy(inv).to(DEV)), q, out)
    torch.cuda.synchronize()
    check(out, q, positions_of(P, C)[None], inv, [0] * 64, False)


def pools(num_pages, hkv, fp8, gen):
    shape = (num_pages, hkv, 16, 128)
    if not fp8:
        return [torch.randn(shape, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2)] + [None, None]
    codes = [torch.randint(0, 120, shape, generator=gen, device=DEV, dtype=torch.int32).to(torch.uint8) for _ in range(2)]
    return codes + [0.004 + 0.02 * torch.rand(hkv, generator=gen, device=DEV) for _ in range(2)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", CASES + [([0, 40, 3], [400, 16, 29], 8, 2, 128, None, False, False)])
def test_append_equals_rotation_and_append(case, fp8):
    """Bit for bit the pages and queries of s2l_rope_qk followed by s2l_kv_append: pages compared whole."""
    P, C, hq, hkv, rot, sections, cyclic, adjacent = case
    print(f"[rope append] {case} fp8={fp8}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(5)
    T = sum(C)
    axes = None if sections is None else s2l.rope_pair_axes(sections, cyclic)
    rope = s2l.Rope(torch.from_numpy(freqs(rot // 2)).to(DEV), positions_for(case, gen)[0], axes, adjacent)
    need = [(p + c + 15) // 16 for p, c in zip(P, C)]
    order = np.random.default_rng(5).permutation(sum(need) + 2)
    tables = np.full((len(P), max(need)), -1, np.int32)
    at = 0
    for r, n in enumerate(need):
        tables[r, :n] = order[at:at + n]
        at += n
    kp, vp, ks, vs = pools(sum(need) + 2, hkv, fp8, gen)
    batch = s2l.Batch(P, C, tables)
    qkv = rows(gen, T, hq + 2 * hkv)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    cache, ref = s2l.PagedKVCache(kp.clone(), vp.clone(), ks, vs), s2l.PagedKVCache(kp, vp, ks, vs)
    q_out, q_ref, k_ref = torch.empty_like(q.contiguous()), torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())
    s2l.s2l_rope_kv_append(cache, batch, rope, q, q_out, k, v)
    s2l.s2l_rope_qk(batch, rope, q, q_ref, k, k_ref)
    s2l.s2l_kv_append(ref, batch, k_ref, v.contiguous())
    torch.cuda.synchronize()
    assert same(q_out, q_ref) and same(cache.k_pages, ref.k_pages) and same(cache.v_pages, ref.v_pages)
    # keys and values alone
    alone = s2l.PagedKVCache(*pools(sum(need) + 2, hkv, fp8, torch.Generator(device=DEV).manual_seed(6))[:2], ks, vs)
    s2l.s2l_rope_kv_append(alone, batch, rope, None, None, k, v)
    s2l.s2l_kv_append(ref, batch, k_ref, v.contiguous())
    out = [torch.zeros((sum(P) + T, hkv, 128), dtype=kp.dtype, device=DEV) for _ in range(4)]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(np.add(P, C))]), dtype=torch.int32, device=DEV)
    s2l.s2l_kv_gather(alone, batch, 1, cu, out[0], out[1])
    s2l.s2l_kv_gather(ref, batch, 1, cu, out[2], out[3])
    torch.cuda.synchronize()
    new = np.concatenate([cu.cpu().numpy()[r] + p + np.arange(c) for r, (p, c) in enumerate(zip(P, C))]).astype(int)
    assert same(out[0][new], out[2][new]) and same(out[1][new], out[3][new])


def test_values_that_are_not_finite_stay_in_their_pair():
    inv = freqs(64)
    q = rows(torch.Generator(device=DEV).manual_seed(7), 4, 2)
    clean = torch.empty_like(q)
    batch, rope = s2l.Batch([3], [4], np.zeros((1, 1), np.int32)), s2l.Rope(torch.from_numpy(inv).to(DEV))
    s2l.s2l_rope_qk(batch, rope, q, clean)
    bad = q.clone()
    bad[1, 0, 5], bad[2, 1, 70] = float("nan"), float("inf")
    out = torch.empty_like(q)
    s2l.s2l_rope_qk(batch, rope, bad, out)
    torch.cuda.synchronize()
    hit = torch.zeros(q.shape, dtype=torch.bool, device=DEV)
    hit[1, 0, [5, 69]] = hit[2, 1, [6, 70]] = True
    assert not bool(torch.isfinite(out[hit]).any()) and same(out[~hit], clean[~hit])


def test_pages_past_four_gib():
    """Pages of a pool above 2^32 bytes, as the same call on a small pool."""
    gen = torch.Generator(device=DEV).manual_seed(8)
    hkv, C = 8, 50
    far = (1 << 32) // (hkv * 16 * 128 * 2) + 5          # beyond 4 GiB
    small = np.arange(4, dtype=np.int32)[None]
    big = np.array([[far, 2, far + 1, far - 7]], np.int32)
    k, v = rows(gen, C, hkv), rows(gen, C, hkv)
    rope = s2l.Rope(torch.from_numpy(freqs(64)).to(DEV))
    got = []
    for tables, n in ((small, 4), (big, far + 2)):
        cache = s2l.PagedKVCache(*(torch.empty((n, hkv, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
        cache.k_pages[tables[0]] = 0
        cache.v_pages[tables[0]] = 0
        s2l.s2l_rope_kv_append(cache, s2l.Batch([9], [C], tables), rope, None, None, k, v)
        torch.cuda.synchronize()
        got.append([cache.k_pages[tables[0]].clone(), cache.v_pages[tables[0]].clone()])
        del cache
    assert same(got[0][0], got[1][0]) and same(got[0][1], got[1][1])
    assert bool((got[0][0] != 0).any())


def test_graph_replays_and_streams():
    gen = torch.Generator(device=DEV).manual_seed(9)
    P, C, hq, hkv = [100, 7], [40, 1], 8, 2
    T = sum(C)
    tables = np.random.default_rng(9).permutation(20).astype(np.int32).reshape(2, 10)
    cache = s2l.PagedKVCache(*(torch.zeros((20, hkv, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    batch, rope = s2l.Batch(P, C, tables), s2l.Rope(torch.from_numpy(freqs(64)).to(DEV))
    q, k, v = rows(gen, T, hq), rows(gen, T, hkv), rows(gen, T, hkv)
    q_out = torch.empty_like(q)
    s2l.s2l_rope_kv_append(cache, batch, rope, q, q_out, k, v)
    torch.cuda.synchronize()
    ref = [t.clone() for t in (q_out, cache.k_pages, cache.v_pages)]
    stream, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(g, stream=stream):
            s2l.s2l_rope_kv_append(cache, batch, rope, q, q_out, k, v, stream)
    for _ in range(3):
        for t in (q_out, cache.k_pages, cache.v_pages):
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            g.replay()
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip((q_out, cache.k_pages, cache.v_pages), ref))


def test_plain_calls_are_marshalled_natively(monkeypatch):
    """None of these calls needs the ctypes path (about 15 us more); positions of one axis in either form."""
    gen = torch.Generator(device=DEV).manual_seed(10)
    P, C, hq, hkv = [3, 40], [5, 1], 4, 2
    T = sum(C)
    batch = s2l.Batch(P, C, np.arange(8, dtype=np.int32).reshape(2, 4))
    cache = s2l.PagedKVCache(*(torch.zeros((8, hkv, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    qkv = rows(gen, T, hq + 2 * hkv)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    pos = torch.randint(0, 99, (3, T), generator=gen, device=DEV, dtype=torch.int32)
    inv = torch.from_numpy(freqs(64)).to(DEV)
    ropes = [s2l.Rope(inv), s2l.Rope(inv, pos[0]), s2l.Rope(inv, pos[:1]), s2l.Rope(inv, pos, s2l.rope_pair_axes((24, 20, 20)), True, 0.5)]

    def both(rope):
        q_out, k_out, q2 = (torch.zeros((T, n, 128), dtype=torch.bfloat16, device=DEV) for n in (hq, hkv, hq))
        s2l.s2l_rope_qk(batch, rope, q, q_out, k, k_out)
        s2l.s2l_rope_kv_append(cache, batch, rope, q, q2, k, v)
        torch.cuda.synchronize()
        assert same(q_out, q2)
        return [q_out, k_out, cache.k_pages.clone()]

    states = torch.randn((3, hq, 128, 128), generator=gen, device=DEV)
    slots = torch.tensor([0, 1], dtype=torch.int32, device=DEV)

    def linear():
        s = states.clone()
        out = torch.zeros((T, hq, 128), dtype=torch.bfloat16, device=DEV)
        s2l.s2l_linear_attn(s2l.LinearState(s, -torch.ones(hq, device=DEV), slots, slots), batch, q, k, v, 0.1, out, None)
        torch.cuda.synchronize()
        return [out, s]

    native = s2l._load_native()
    with monkeypatch.context() as m:   # the general path
        m.setattr(s2l, "_native", s2l._lib._NoBinding)
        ref = [both(r) for r in ropes] + [linear()]
    assert s2l._native is native
    with monkeypatch.context() as m:
        m.setattr(s2l._lib, "call", None)
        got = [both(r) for r in ropes] + [linear()]
    assert all(same(a, b) for x, y in zip(ref, got) for a, b in zip(x, y))
    assert same(got[1][0], got[2][0]) and not same(got[0][0], got[1][0])


def test_append_rotates_queries_in_place():
    """q_out may be q: a view of the projected row that k and v are views of too."""
    gen = torch.Generator(device=DEV).manual_seed(11)
    P, C, hq, hkv = [7, 0], [40, 9], 8, 2
    T = sum(C)
    batch, rope = s2l.Batch(P, C, np.arange(8, dtype=np.int32).reshape(2, 4)), s2l.Rope(torch.from_numpy(freqs(64)).to(DEV))
    caches = [s2l.PagedKVCache(*(torch.zeros((8, hkv, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))) for _ in range(2)]
    qkv = rows(gen, T, hq + 2 * hkv, pad=1)
    before, out = qkv.clone(), torch.empty((T, hq, 128), dtype=torch.bfloat16, device=DEV)
    views = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    s2l.s2l_rope_kv_append(caches[0], batch, rope, views[0], out, views[1], views[2])
    s2l.s2l_rope_kv_append(caches[1], batch, rope, views[0], views[0], views[1], views[2])
    torch.cuda.synchronize()
    assert same(qkv[:T, :hq], out) and same(qkv[:, hq:], before[:, hq:]) and same(qkv[T:], before[T:])
    assert same(caches[0].k_pages, caches[1].k_pages) and same(caches[0].v_pages, caches[1].v_pages)


def test_wide_rows_take_two_heads_a_lane():
    """Enough rows for the form with two heads a lane, head counts that fill its last group in part."""
    gen = torch.Generator(device=DEV).manual_seed(12)
    for hq, hkv in ((17, 2), (9, 9), (1, 33)):
        T = 9000
        inv = freqs(48)
        q, k = rows(gen, T, hq), rows(gen, T, hkv)
        q_out, k_out = torch.zeros_like(q), torch.zeros_like(k)
        P, C = [5, 1000], [8000, 1000]
        s2l.s2l_rope_qk(s2l.Batch(P, C, np.zeros((2, 1), np.int32)), s2l.Rope(torch.from_numpy(inv).to(DEV)), q, q_out, k, k_out)
        torch.cuda.synchronize()
        pick = torch.arange(0, T, 97, device=DEV)
        pos = positions_of(P, C)[None][:, ::97]
        check(q_out[pick], q[pick], pos, inv, [0] * 48, False)
        check(k_out[pick], k[pick], pos, inv, [0] * 48, False)
