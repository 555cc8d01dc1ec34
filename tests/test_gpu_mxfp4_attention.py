"""GPU: attention over MXFP4 pages against the oracle, in every layout, with the bound of the other page
types (the pages' values are exact in bf16, so the arithmetic is the same)."""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
import workloads
from oracle import mxfp4
from oracle.paged_kv import bf16_bits_to_f32
from tests.gpu_util import DEV, LOG2E, SCALE, assert_attention_close, bf16_to_f64, plant_dots_for, to_bf16
from tests.mxfp4_util import MxSetup, mx_case, quantised_bits, slots

pytestmark = pytest.mark.gpu

LAYOUTS = [(16, 1), (128, 1), (128, 2), (256, 1)]
SPLIT = dict(target_items=1 << 20, min_split_keys=64, max_splits=16)


def opts_of(layout, split=False):
    return s2l.plan_opts(tile_cols=layout[0], key_halves=layout[1], **(SPLIT if split else {}))


@pytest.mark.parametrize("hq,hkv", [(2, 2), (7, 1), (32, 8), (16, 1)])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_layouts(layout, split, hq, hkv):
    """Whole tiles, a token more, single tokens, ranges that end inside pages and tiles, and an empty request."""
    tq = layout[0] // (hq // hkv)
    case = mx_case("mx", [500, 0, 64, 1003, 37, 15], [tq + 1, 1, tq, 1, 0, 2], hq, hkv, seed=60)
    s = MxSetup(case)
    s.append()
    out, lse = s.attention(opts_of(layout, split))
    assert s.plan.tile_cols == layout[0]
    assert_attention_close(case, out, lse, s.oracle(), what=f"{layout} split={split}")


@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 257])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_short_ranges(layout, n):
    """One token that sees n keys, and a whole chunk of n."""
    case = mx_case("short", [n - 1, 0], [1, n], 4, 2, seed=61)
    s = MxSetup(case)
    s.append()
    out, lse = s.attention(opts_of(layout))
    assert_attention_close(case, out, lse, s.oracle(), what=f"{n} keys, {layout}")


HEADS = [(8, 8), (16, 8), (24, 8), (32, 8), (64, 8), (12, 4), (6, 1), (40, 8), (48, 4)]


@pytest.mark.parametrize("seed", range(20))
def test_random_batches(seed):
    rng = np.random.default_rng(70 + seed)
    R = int(rng.integers(1, 6))
    P = [int(rng.choice([0, 16 * rng.integers(1, 100), rng.integers(1, 2000)])) for _ in range(R)]
    decode = rng.random() < 0.4
    C = [int(rng.integers(1, 3)) if decode else int(np.exp(rng.uniform(0, 6))) for _ in range(R)]
    hq, hkv = HEADS[int(rng.integers(len(HEADS)))]
    layout = [None, (128, 1), (128, 2), (256, 1)][int(rng.integers(4))]
    split = bool(rng.random() < 0.5)
    kw = {} if layout is None else dict(tile_cols=layout[0], key_halves=layout[1])
    case = mx_case(f"mxfuzz{seed}", P, C, hq, hkv, seed=seed)
    s = MxSetup(case)
    s.append()
    out, lse = s.attention(s2l.plan_opts(**kw, **(SPLIT if split else {})))
    assert_attention_close(case, out, lse, s.oracle(), what=f"seed {seed}: {P} {C} {hq}/{hkv} {layout} split={split}")


@pytest.mark.parametrize("layout", LAYOUTS)
def test_blocks_of_every_size(layout):
    """Values' blocks from 2^-60 to 2^60 side by side in a row, keys' from 2^-20 to 2: each block by its own scale."""
    hq, hkv = 4, 2
    case = mx_case("sizes", [333], [5], hq, hkv, seed=62)
    rng = np.random.default_rng(62)
    for name, lo, hi in (("k_full_bits", -20, 2), ("v_full_bits", -60, 60)):
        x = bf16_bits_to_f32(getattr(case, name)).astype(np.float64)
        size = 2.0 ** (np.repeat(rng.integers(lo, hi, x.shape[1:-1] + (4,)), 32, -1))
        setattr(case, name, quantised_bits((x * size).astype(np.float32).view(np.uint32) >> 16))
    s = MxSetup(case)
    s.append()
    out, lse = s.attention(opts_of(layout))
    o, l, a, b = s.oracle()
    u = 2.0 ** -8       # the bound of assert_attention_close, at values of any size
    err = np.abs(bf16_to_f64(out) - o)
    assert (err <= u * np.abs(o) + 2.02 * u * b + 2.0 ** -16 * a).all()
    assert (np.abs(lse.cpu().numpy() - l) <= u + 1e-4 * (1 + np.abs(l))).all()


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_scores_that_rise_past_the_reference(layout, split):
    """Planted keys each 72 log2 units above the ones before, so the reference has to be raised: the largest
    score of keys from 64 on is checked to be more than 64 above those of the first 64 of each range."""
    hq, hkv = 8, 2
    case = mx_case("planted", [2000], [2], hq, hkv, seed=63, plant_dots=plant_dots_for(72.0, 4), plant_twin_gap=1 / (SCALE * LOG2E))
    s = MxSetup(case)
    s.append()
    q, k = bf16_bits_to_f32(case.q_bits).astype(np.float64), bf16_bits_to_f32(case.k_full_bits).astype(np.float64)
    score = SCALE * LOG2E * (k[:, 0] @ q[1, 0])
    assert score[64:].max() - score[:64].max() > 64
    out, lse = s.attention(opts_of(layout, split))
    assert_attention_close(case, out, lse, s.oracle(), what=f"{layout}")


@pytest.mark.parametrize("layout", LAYOUTS)
def test_queries_far_below_their_block(layout):
    """Dims with queries 2000 times the others, over which all keys are zero: the scores come from the small ones.
    Tiles of 128 and 256 columns take a query within 2^-13 of its block's largest, so a score is off by at most
    d = 2^-13 scale sum_blocks largest sum |K|, a weight by e^(2 d) - 1 of itself; those of 16 columns take it whole."""
    hq, hkv = 8, 2
    case = mx_case("outliers", [400], [2], hq, hkv, seed=69, sigma=1.0)
    q, k = bf16_bits_to_f32(case.q_bits).reshape(2, hq, 4, 32), bf16_bits_to_f32(case.k_full_bits)
    q[:, :, :3, 5] = 2000 * np.sign(q[:, :, :3, 5])
    k[:, :, [5, 37, 69]] = 0
    case.q_bits, case.k_full_bits = workloads.bf16_bits(q.reshape(2, hq, 128)), quantised_bits(workloads.bf16_bits(k))
    s = MxSetup(case)
    s.append()
    out, lse = s.attention(opts_of(layout))
    o, l, a, b = s.oracle()
    kept = np.abs(bf16_bits_to_f32(case.k_full_bits).astype(np.float64)).reshape(-1, hkv, 4, 32).sum(-1)      # [keys][hkv][4]
    top = np.abs(q.astype(np.float64)).max(-1).reshape(2, hkv, hq // hkv, 4)
    d = 0 if layout[0] == 16 else 2.0 ** -13 * SCALE * np.einsum("tgjb,kgb->tgjk", top, kept).max(-1).reshape(2, hq)
    u = 2.0 ** -8
    err = np.abs(bf16_to_f64(out) - o)
    assert (err <= u * np.abs(o) + (2.02 * u + np.expm1(2 * np.asarray(d))[..., None]) * b + 2.0 ** -16 * a + 1e-6).all()
    assert (np.abs(lse.cpu().numpy() - l) <= u + d + 1e-4 * (1 + np.abs(l))).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_a_query_that_is_not_finite(layout, bad):
    """Its own row is NaN; the others of its tile keep their bits."""
    case = mx_case("bad_q", [300], [4], 4, 2, seed=70)
    s = MxSetup(case)
    s.append()
    ref, ref_lse = s.attention(opts_of(layout))
    s.q[2, 1, 77] = bad
    out, lse = s.attention(opts_of(layout))
    assert torch.isnan(out[2, 1]).all() and torch.isnan(lse[2, 1])
    out[2, 1], lse[2, 1] = ref[2, 1], ref_lse[2, 1]
    assert torch.equal(out.view(torch.int16), ref.view(torch.int16)) and torch.equal(lse, ref_lse)


@pytest.mark.parametrize("scale", [2.0 ** -120, 1e-30, 1e-4, 0.7, 1.9, 1.0e3])
@pytest.mark.parametrize("layout", [(128, 1), (256, 1)])
def test_other_softmax_scales(layout, scale):
    """Factors of every mantissa and size, with queries of sizes from 2^-100 to 2 (scores up to thousands)."""
    case = mx_case("scales", [130], [3], 2, 2, seed=71)
    q = bf16_bits_to_f32(case.q_bits)
    q[0] *= np.float32(2.0 ** -100)
    q[1] *= np.float32(4 / max(scale, 1e-3) / 8)
    case.q_bits = workloads.bf16_bits(q)
    s = MxSetup(case)
    s.append()
    out, lse = s.attention(opts_of(layout), scale=scale)
    o, l, a, b = s.oracle(scale=scale)
    keys = np.abs(bf16_bits_to_f32(case.k_full_bits).astype(np.float64)).reshape(-1, 2, 4, 32).sum(-1)
    top = np.abs(bf16_bits_to_f32(case.q_bits).astype(np.float64)).reshape(3, 2, 4, 32).max(-1)
    # the queries' terms, and fp32 sums of products up to the largest score
    d = (2.0 ** -13 + 2.0 ** -18) * scale * np.einsum("tgb,kgb->tgk", top, keys).max(-1)
    u = 2.0 ** -8
    err = np.abs(bf16_to_f64(out) - o)
    assert (err <= u * np.abs(o) + (2.02 * u + np.expm1(2 * d)[..., None]) * b + 2.0 ** -16 * a + 1e-6).all()
    assert (np.abs(lse.cpu().numpy() - l) <= u + d + 1e-4 * (1 + np.abs(l))).all()


@pytest.mark.parametrize("layout", LAYOUTS)
def test_what_lies_behind_the_sequence_has_no_effect(layout):
    """Any bytes in the slots behind each sequence's end, in its last page and in the pages after, among them scale
    bytes that stand for NaN or pass every range: the bits stay."""
    case = mx_case("behind", [70, 5, 0], [3, 20, 1], 4, 2, seed=72)
    s = MxSetup(case)
    s.append()
    ref, ref_lse = s.attention(opts_of(layout))
    rng = np.random.default_rng(72)
    for pool in (s.cache.k_pages, s.cache.v_pages):
        host = pool.cpu().numpy()
        host[case.poison_page] = rng.integers(0, 256, host[0].shape)
        for r in range(3):
            n = int(case.prefix_lens[r] + case.chunk_lens[r])
            page, slot = slots(case.block_tables, r, range(n, -(-n // 16) * 16))
            for p, i in zip(page, slot):
                host[p, :, 64 * i:64 * i + 64] = rng.integers(0, 256, (2, 64))
                host[p, :, 1024 + 4 * i:1028 + 4 * i] = rng.integers(250, 256, (2, 4))
        pool.copy_(torch.from_numpy(host))
    out, lse = s.attention(opts_of(layout))
    assert torch.equal(out.view(torch.int16), ref.view(torch.int16)) and torch.equal(lse, ref_lse)


@pytest.mark.parametrize("offset", [1, 4])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_q_and_out_of_a_view_between_16_byte_boundaries(layout, offset):
    for hq, hkv in ((2, 2), (7, 1)):
        tq = layout[0] // (hq // hkv)
        case = mx_case("views", [100, 0], [tq + 1, tq], hq, hkv, seed=73)
        s = MxSetup(case)
        s.append()
        T = case.total_tokens
        ref, ref_lse = s.attention(opts_of(layout))
        n = T * hq * 128
        q = torch.empty(n + offset, dtype=torch.bfloat16, device=DEV)[offset:].view(T, hq, 128).copy_(s.q)
        out = torch.full((n + offset,), float("nan"), dtype=torch.bfloat16, device=DEV)[offset:].view(T, hq, 128)
        lse = torch.empty_like(ref_lse)
        s2l.s2l_chunk_prefill_attn(s.cache, s.batch, q, hq, SCALE, out, lse, s.plan, s._ws)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), ref.view(torch.int16)) and torch.equal(lse, ref_lse)


@pytest.mark.parametrize("R,hi", [(70, 4096), (100, 900), (300, 64)])
def test_decode_batches_of_every_residency(R, hi):
    """Binned, sorted and equal items, long and short, so that one workgroup a CU and two are run; a sample of rows."""
    rng = np.random.default_rng(R)
    P = rng.integers(1, hi, R)
    case = mx_case("rounds", P, [1] * R, 32, 8, seed=R)
    s = MxSetup(case)
    s.append()
    out, lse = s.attention()
    rows = {r: [0] for r in rng.choice(R, 24, replace=False).tolist() + [int(P.argmax()), int(P.argmin())]}
    assert s.plan.tile_cols == 16
    assert_attention_close(case, out, lse, s.oracle(sample_rows=rows), rows, what=f"{R} rows")


def nan_block(pool, tables, r, key, head, block):
    page, slot = slots(tables, r, [key])
    pool[page[0], head, 1024 + 4 * slot[0] + block] = 255


PLANS = [dict(target_items=1), dict(), dict(target_items=1 << 20, min_split_keys=64, max_splits=64)]


@pytest.mark.parametrize("layout", LAYOUTS)
def test_a_nan_of_v_reaches_the_rows_and_dims_that_see_it(layout):
    """In a cached key, in the middle of the chunk, in its last key, and in keys behind the sequence that share its
    page: the rows that see the key get NaN in the block's 32 dims; everything else keeps its bits."""
    hq, hkv, P, C = 4, 2, 700, 6
    case = mx_case("nan_v", [P, 64], [C, 3], hq, hkv, seed=64)
    s = MxSetup(case)
    s.append()
    for key, block in ((300, 1), (P + 2, 3), (P + C - 1, 0), (P + C, 2), (0, 2)):
        for plan in PLANS:
            opts = s2l.plan_opts(tile_cols=layout[0], key_halves=layout[1], **plan)
            clean, clean_lse = s.attention(opts)
            saved = s.cache.v_pages.clone()
            nan_block(s.cache.v_pages, case.block_tables, 0, min(key, 707), 1, block)
            out, lse = s.attention(opts)
            s.cache.v_pages.copy_(saved)
            seen = min(max(0, key - P), C)
            what = f"key {key} block {block} {plan}"
            dims = slice(32 * block, 32 * block + 32)
            assert torch.isnan(out[seen:C, 2:, dims]).all(), what
            out[seen:C, 2:, dims] = clean[seen:C, 2:, dims]
            assert torch.equal(out.view(torch.int16), clean.view(torch.int16)) and torch.equal(lse, clean_lse), what


@pytest.mark.parametrize("layout", LAYOUTS)
def test_a_nan_of_k_reaches_the_rows_that_see_it(layout):
    hq, hkv, P, C = 4, 2, 700, 6
    case = mx_case("nan_k", [P, 64], [C, 3], hq, hkv, seed=65)
    s = MxSetup(case)
    s.append()
    for key in (300, P + 2, P + C - 1):
        for plan in PLANS:
            opts = s2l.plan_opts(tile_cols=layout[0], key_halves=layout[1], **plan)
            clean, clean_lse = s.attention(opts)
            saved = s.cache.k_pages.clone()
            nan_block(s.cache.k_pages, case.block_tables, 0, key, 1, 2)
            out, lse = s.attention(opts)
            s.cache.k_pages.copy_(saved)
            seen = max(0, key - P)
            assert torch.isnan(out[seen:C, 2:]).all() and torch.isnan(lse[seen:C, 2:]).all(), (key, plan)
            out[seen:C, 2:], lse[seen:C, 2:] = clean[seen:C, 2:], clean_lse[seen:C, 2:]
            assert torch.equal(out.view(torch.int16), clean.view(torch.int16)) and torch.equal(lse, clean_lse), (key, plan)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_pages_past_four_gibibytes(layout):
    """The same bits from pools of 4.4 GB whose even logical pages lie past 4 GiB."""
    case = mx_case("far", [700, 33], [40, 3], 8, 2, seed=66)
    near = MxSetup(case)
    near.append()
    ref, ref_lse = near.attention(opts_of(layout, True))
    base = (1 << 32) // (2 * mxfp4.RUN) + 1
    lp = np.arange(case.block_tables.shape[1])[None]
    tables = np.where(lp % 2 == 0, case.block_tables + base, case.block_tables).astype(np.int32)
    pools = [torch.zeros((base + case.num_pages, 2, mxfp4.RUN), dtype=torch.uint8, device=DEV) for _ in range(2)]
    for pool, src in zip(pools, (near.cache.k_pages, near.cache.v_pages)):
        pool[:case.num_pages] = src
        pool[base:] = src
    far = MxSetup(case)
    far.batch, far.cache = s2l.Batch(case.prefix_lens, case.chunk_lens, tables), s2l.PagedKVCache(*pools)
    out, lse = far.attention(opts_of(layout, True))
    assert torch.equal(out.view(torch.int16), ref.view(torch.int16)) and torch.equal(lse, ref_lse)


def test_the_calls_that_plan_append_or_split_by_themselves():
    """Append with attention, attention without a workspace, and the two launches apart: the bits of the plain calls."""
    case = mx_case("calls", [320, 0, 48], [40, 17, 16], 16, 4, seed=67)
    s = MxSetup(case)
    s.append()
    hq, T = case.num_q_heads, case.total_tokens
    ref, ref_lse = s.attention()
    two, two_lse = s.attention(use_main_and_reduce=True)
    assert torch.equal(two, ref) and torch.equal(two_lse, ref_lse)
    out, lse = torch.empty_like(ref), torch.empty_like(ref_lse)
    s2l.s2l_chunk_prefill_attn_noalloc(s.cache, s.batch, s.q, hq, SCALE, out, lse)
    torch.cuda.synchronize()
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    other = MxSetup(case)
    fused = s2l.s2l_append_chunk_prefill_attn(other.cache, other.batch, to_bf16(s.k_new), to_bf16(s.v_new), s.q, hq, SCALE, out.zero_(),
                                              lse.zero_(), s.plan, s._ws)
    torch.cuda.synchronize()
    assert not fused and torch.equal(out, ref) and torch.equal(lse, ref_lse)
    assert torch.equal(other.cache.k_pages, s.cache.k_pages) and torch.equal(other.cache.v_pages, s.cache.v_pages)
    with pytest.raises(s2l.S2LError, match="ENOTSUP"):
        s2l.s2l_chunk_prefill_attn_q8(s.cache, s.batch, s.q, hq, SCALE, out, lse, s.plan, s._ws)


def test_device_lengths_that_need_more_than_was_planned():
    """The outputs are NaN throughout, as with the other page types."""
    case = mx_case("status", [64], [1], 4, 2, seed=68)
    s = MxSetup(case)
    s.append()
    s.batch.chunk_lens.fill_(500)
    out, lse = s.attention()
    assert torch.isnan(out).all() and torch.isnan(lse).all()
