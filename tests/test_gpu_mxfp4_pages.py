"""GPU: MXFP4 pages written, read back, gathered and swapped, bit for bit against the definition."""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from oracle import mxfp4
from oracle.fp8_e4m3 import e4m3_decode
from tests.gpu_util import DEV, from_bf16, to_bf16
from tests.mxfp4_util import slots, to_f64

pytestmark = pytest.mark.gpu

BATCHES = [  # prefixes, chunks, kv heads
    ([2047], [1], 8),
    ([0], [1], 1),
    ([5, 16, 0, 33, 15], [3, 16, 0, 70, 2], 2),
    ([0, 31], [130, 1], 5),
]


def tables_for(P, C, rng):
    need = [-(-(p + c) // 16) for p, c in zip(P, C)]
    order = rng.permutation(sum(need) + 2)
    tables, at = np.zeros((len(P), max(max(need), 1)), np.int32), 0
    for r, n in enumerate(need):
        tables[r, :n] = order[at:at + n]
        at += n
    return tables, sum(need) + 2


def pools(pages, hkv, rng):
    host = [rng.integers(0, 256, (pages, hkv, mxfp4.RUN), dtype=np.uint8) for _ in range(2)]
    return host, s2l.PagedKVCache(*(torch.from_numpy(p.copy()).to(DEV) for p in host))


def draw_rows(T, hkv, rng):
    """Rows of every size that bf16 has, blocks of zeros, denormals, and some that are not finite."""
    x = rng.standard_normal((T, hkv, 128)) * 2.0 ** rng.integers(-12, 12, (T, hkv, 1))
    x[rng.random((T, hkv, 128)) < 0.1] = 0
    kind = np.repeat(rng.random((T, hkv, 4)), 32, -1)
    x = np.where(kind < 0.05, 0.0, np.where(kind < 0.1, x * 2.0 ** -128, np.where(kind < 0.15, x * 2.0 ** 112, x)))
    bits = np.clip(x, -3.38e38, 3.38e38).astype(np.float32).view(np.uint32) >> 16
    odd = rng.random(bits.shape)
    return np.where(odd < 0.001, 0x7FC0, np.where(odd < 0.002, 0xFF80, bits)).astype(np.uint16)


def store(host, tables, P, C, rows):
    at = 0
    for r, (p, c) in enumerate(zip(P, C)):
        page, slot = slots(tables, r, range(p, p + c))
        mxfp4.store(host, page, slot, to_f64(rows[at:at + c]))
        at += c


@pytest.mark.parametrize("P,C,hkv", BATCHES)
def test_append_writes_its_slots_and_nothing_else(P, C, hkv):
    rng = np.random.default_rng(sum(P) + sum(C))
    tables, pages = tables_for(P, C, rng)
    host, cache = pools(pages, hkv, rng)
    rows = [draw_rows(sum(C), hkv, rng) for _ in range(2)]
    s2l.s2l_kv_append(cache, s2l.Batch(P, C, tables), to_bf16(rows[0]), to_bf16(rows[1]))
    torch.cuda.synchronize()
    for pool, h, x in zip((cache.k_pages, cache.v_pages), host, rows):
        store(h, tables, P, C, x)
        assert np.array_equal(pool.cpu().numpy(), h)


def test_append_of_every_bf16_value():
    """Each bf16 pattern in a block of its own (with a larger neighbour in half of them), so every exponent,
    every rounding and every value that is not finite."""
    bits = np.zeros((1024, 2, 128), np.uint16)
    value = np.arange(65536, dtype=np.uint32)
    block = bits.reshape(-1, 32)                     # 8192 blocks a round
    for part in range(8):
        v = value[part * 8192:(part + 1) * 8192]
        block[:] = 0
        block[:, 5] = v
        block[::2, 17] = np.minimum((v[::2] & 0x7FFF) + 0x0155, 0x7F7F)     # 2.67 binades up
        pages = 64
        host, cache = pools(pages, 2, np.random.default_rng(part))
        tables = np.random.default_rng(part).permutation(pages).astype(np.int32)[None]
        s2l.s2l_kv_append(cache, s2l.Batch([0], [1024], tables), to_bf16(bits), to_bf16(bits[::-1].copy()))
        torch.cuda.synchronize()
        store(host[0], tables, [0], [1024], bits)
        store(host[1], tables, [0], [1024], bits[::-1])
        assert np.array_equal(cache.k_pages.cpu().numpy(), host[0]) and np.array_equal(cache.v_pages.cpu().numpy(), host[1]), part


PARTS = {s2l.S2L_READ_PREFIX: lambda p, c: range(p), s2l.S2L_READ_ALL: lambda p, c: range(p + c), s2l.S2L_READ_CHUNK: lambda p, c: range(p, p + c)}


@pytest.mark.parametrize("kind", ["bf16", "fp8", "mxfp4"])
@pytest.mark.parametrize("P,C,hkv", BATCHES)
def test_read_gives_the_values(P, C, hkv, kind):
    """Each part, with rows in an order of their own, rows cut off at the end of the output and rows before it."""
    rng = np.random.default_rng(7 * sum(P) + sum(C))
    tables, pages = tables_for(P, C, rng)
    if kind == "mxfp4":
        host, cache = pools(pages, hkv, rng)
        for h, dev in zip(host, (cache.k_pages, cache.v_pages)):
            at = h[..., 1024:]
            at[(at == 253) | (at == 254)] = 127      # values past bf16's range
            dev.copy_(torch.from_numpy(h))
        values = [lambda page, slot, h=h: mxfp4.load(h, page, slot)[1] for h in host]
    elif kind == "bf16":
        host = [draw_rows(pages * hkv, 16, rng).reshape(pages, hkv, 16, 128) for _ in range(2)]
        cache = s2l.PagedKVCache(*(to_bf16(h) for h in host))
        values = [lambda page, slot, h=h: to_f64(h[page, :, slot]) for h in host]
    else:
        host = [rng.integers(0, 256, (pages, hkv, 16, 128), dtype=np.uint8) for _ in range(2)]
        scale = [np.exp(rng.standard_normal(hkv)).astype(np.float32) for _ in range(2)]
        cache = s2l.PagedKVCache(*(torch.from_numpy(h).to(DEV) for h in host), *(torch.from_numpy(x).to(DEV) for x in scale))
        values = [lambda page, slot, h=h, x=x: (e4m3_decode(h[page, :, slot]).astype(np.float32) * x[:, None]).astype(np.float64)
                  for h, x in zip(host, scale)]
    batch = s2l.Batch(P, C, tables)
    for part, positions in PARTS.items():
        n = [len(positions(p, c)) for p, c in zip(P, C)]
        order = rng.permutation(len(P))
        cu, at = np.zeros(len(P), np.int32), -2      # two rows of the first request are before the output
        for r in order:
            cu[r] = at
            at += n[r] + 1
        rows = max(at - 3, 1)                        # the last request's last row or two behind it
        want = [np.full((rows, hkv, 128), 7.0) for _ in range(2)]
        for w, of in zip(want, values):
            for r, (p, c) in enumerate(zip(P, C)):
                if n[r] == 0:
                    continue
                x = of(*slots(tables, r, positions(p, c)))
                for i in range(n[r]):
                    if 0 <= cu[r] + i < rows:
                        w[cu[r] + i] = x[i]
        k, v = (torch.full((rows, hkv, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        s2l.s2l_kv_read(cache, batch, part, torch.from_numpy(cu).to(DEV), k, v)
        torch.cuda.synchronize()
        for got, w in zip((k, v), want):
            # one rounding to bf16 at most (e4m3 times its scale): none of the other two
            w = torch.from_numpy(w).to(torch.float32).to(torch.bfloat16).to(DEV)
            assert torch.equal(torch.isnan(got), torch.isnan(w)), (part, kind)
            assert torch.equal(got.nan_to_num(0), w.nan_to_num(0)), (part, kind)


@pytest.mark.parametrize("P", [3201, 6655])
def test_read_of_more_than_caches_hold(P):
    """Outputs of 105 and 218 MB, where values are stored past the caches, from pages that requests share, and of a request alone."""
    rng = np.random.default_rng(P)
    host, cache = pools(40, 8, rng)
    for h, dev in zip(host, (cache.k_pages, cache.v_pages)):
        h[..., 1024:] = rng.integers(100, 140, h[..., 1024:].shape)
        dev.copy_(torch.from_numpy(h))
    tables = rng.integers(0, 40, (8, -(-P // 16))).astype(np.int32)
    whole = [mxfp4.load(h, np.repeat(np.arange(40), 16), np.tile(np.arange(16), 40))[1] for h in host]    # of every page
    whole = [torch.from_numpy(w).to(torch.float32).to(torch.bfloat16).to(DEV).view(40, 16, 8, 128) for w in whole]
    for R in (8, 1):
        batch = s2l.Batch([P] * R, [0] * R, tables[:R])
        k, v = (torch.full((R * P, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        s2l.s2l_kv_read(cache, batch, s2l.S2L_READ_PREFIX, torch.arange(R, device=DEV).int() * P, k, v)
        torch.cuda.synchronize()
        for got, w in zip((k, v), whole):
            for r in range(R):
                want = w[torch.from_numpy(tables[r].astype(np.int64)).to(DEV)].reshape(-1, 8, 128)[:P]
                assert torch.equal(got[r * P:(r + 1) * P], want), (R, r)


def test_read_of_nothing():
    cache = pools(2, 2, np.random.default_rng(0))[1]
    k = torch.zeros((0, 2, 128), dtype=torch.bfloat16, device=DEV)
    for P, C in (([], []), ([0], [0]), ([16], [4])):
        batch = s2l.Batch(P, C, np.zeros((len(P), 2), np.int32))
        s2l.s2l_kv_read(cache, batch, s2l.S2L_READ_ALL, batch.cu_chunk, k, k)
    torch.cuda.synchronize()


@pytest.mark.parametrize("P,C,hkv", BATCHES)
def test_gather_copies_codes_and_scales(P, C, hkv):
    rng = np.random.default_rng(3 * sum(P) + sum(C))
    tables, pages = tables_for(P, C, rng)
    host, cache = pools(pages, hkv, rng)
    batch = s2l.Batch(P, C, tables)
    for chunk in (0, 1):
        n = [p + chunk * c for p, c in zip(P, C)]
        cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        k, v = (torch.zeros((int(cu[-1]) + 1, hkv, 68), dtype=torch.uint8, device=DEV) for _ in range(2))
        s2l.s2l_kv_gather(cache, batch, chunk, torch.from_numpy(cu).to(DEV), k, v)
        torch.cuda.synchronize()
        for got, h in zip((k, v), host):
            want = [mxfp4.load(h, *slots(tables, r, range(m)))[0] for r, m in enumerate(n) if m]
            assert np.array_equal(got[:-1].cpu().numpy(), np.concatenate(want) if want else got[:-1].cpu().numpy())
            assert not got[-1].any()


@pytest.mark.parametrize("hkv", [1, 8])
def test_swap_moves_whole_pages(hkv):
    rng = np.random.default_rng(hkv)
    host, cache = pools(9, hkv, rng)
    away = [torch.zeros((4, hkv, mxfp4.RUN), dtype=torch.uint8).pin_memory() for _ in range(2)]
    s2l.s2l_kv_swap_out(cache, torch.tensor([[8, 0], [3, 2], [9, 1], [0, 4]], dtype=torch.int32, device=DEV), *away)   # two outside
    torch.cuda.synchronize()
    for a, h in zip(away, host):
        assert np.array_equal(a.numpy()[[0, 2]], h[[8, 3]]) and not a[1].any() and not a[3].any()
    s2l.s2l_kv_swap_in(cache, torch.tensor([[2, 5], [0, 0]], dtype=torch.int32, device=DEV), *away)
    torch.cuda.synchronize()
    for pool, h in zip((cache.k_pages, cache.v_pages), host):
        h[5], h[0] = h[3].copy(), h[8].copy()
        assert np.array_equal(pool.cpu().numpy(), h)


@pytest.mark.parametrize("rot", [16, 64, 96, 128])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rotating_append_is_rotation_then_append(rot, adjacent):
    """Pages of the one call, bit for bit those of the two, with few and with many rows (one head a lane and two)."""
    gen = torch.Generator(device=DEV).manual_seed(rot)
    inv = torch.from_numpy((10000.0 ** -(np.arange(rot // 2) / (rot // 2))).astype(np.float32)).to(DEV)
    rope = s2l.Rope(inv, adjacent=adjacent)
    for P, C, hq, hkv in (([2047], [1], 8, 2), ([5, 0, 30], [33, 0, 21], 0, 5), ([7, 100], [700, 1200], 32, 8)):
        rng = np.random.default_rng(rot)
        tables, pages = tables_for(P, C, rng)
        (_, one), (_, two) = pools(pages, hkv, rng), pools(pages, hkv, np.random.default_rng(0))
        two.k_pages.copy_(one.k_pages), two.v_pages.copy_(one.v_pages)
        batch, T = s2l.Batch(P, C, tables), sum(C)
        qkv = torch.randn((T, hq + 2 * hkv, 128), generator=gen, device=DEV).to(torch.bfloat16)
        qkv[0, -1, 40] = float("nan")
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        q1, q2, k2 = torch.empty((T, hq, 128), dtype=torch.bfloat16, device=DEV), torch.empty((T, hq, 128), dtype=torch.bfloat16, device=DEV), torch.empty((T, hkv, 128), dtype=torch.bfloat16, device=DEV)
        s2l.s2l_rope_kv_append(one, batch, rope, q if hq else None, q1 if hq else None, k, v)
        s2l.s2l_rope_qk(batch, rope, q, q2, k, k2)
        s2l.s2l_kv_append(two, batch, k2, v.contiguous())
        torch.cuda.synchronize()
        assert torch.equal(q1.view(torch.int16), q2.view(torch.int16))
        assert torch.equal(one.k_pages, two.k_pages) and torch.equal(one.v_pages, two.v_pages), (P, C)


def test_pages_past_four_gibibytes():
    """Offsets of codes, scales and rows that pass 32 bits: append, gather and read of pages at the end of pools of
    4.4 GB each."""
    hkv, pages = 8, (1 << 32) // (8 * mxfp4.RUN) + 16
    cache = s2l.PagedKVCache(*(torch.zeros((pages, hkv, mxfp4.RUN), dtype=torch.uint8, device=DEV) for _ in range(2)))
    rng = np.random.default_rng(9)
    tables = np.array([[pages - 1, 3, pages - 9]], np.int32)
    rows = [draw_rows(40, hkv, rng) for _ in range(2)]
    batch = s2l.Batch([3], [40], tables)
    s2l.s2l_kv_append(cache, batch, to_bf16(rows[0]), to_bf16(rows[1]))
    k, v = (torch.zeros((40, hkv, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    s2l.s2l_kv_read(cache, batch, s2l.S2L_READ_CHUNK, batch.cu_chunk, k, v)
    gk, gv = (torch.zeros((43, hkv, 68), dtype=torch.uint8, device=DEV) for _ in range(2))
    s2l.s2l_kv_gather(cache, batch, 1, torch.zeros(2, dtype=torch.int32, device=DEV), gk, gv)
    torch.cuda.synchronize()
    for got, data, x in zip((k, v), (gk, gv), rows):
        codes, scales = mxfp4.quantise(to_f64(x))
        assert np.array_equal(data[3:].cpu().numpy(), np.concatenate([mxfp4.pack(codes), scales], -1))
        want = mxfp4.dequantise(codes, scales)
        got = to_f64(from_bf16(got))
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.nan_to_num(got), np.nan_to_num(want))
