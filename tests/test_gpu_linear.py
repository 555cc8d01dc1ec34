"""GPU: linear attention with a decay against float64, token after token.

Bounds: A and B are the outputs' and states' sums with every product's absolute value (the oracle returns them).
A state of C tokens is C + 1 fp32 steps of two roundings (2^-24 each) and a power of the decay (a few
more): |err| <= (2 C + 16) 2^-24 B.  An output sums 128 of these with fp32 roundings, its factors
that are no bf16 values are two bf16 terms (2^-16 together for two of them), and it is rounded once:
|err| <= 2^-8 |out| + (2^-15 + (2 C + 160) 2^-24) A.
"""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from oracle.linear_attn import linear_attn
from tests.gpu_util import DEV, bf16_to_f64

pytestmark = pytest.mark.gpu
SCALE = 128.0 ** -0.5


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def slopes(hq):
    return (-(2.0 ** (-8.0 * (np.arange(hq) + 1) / hq))).astype(np.float32)


class Step:
    def __init__(self, C, hq, hkv, seed, slot_in=None, slot_out=None, num_slots=None, log_decay=None, P=None):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        R, T = len(C), int(sum(C))
        self.C, self.hq, self.hkv, self.T = [int(c) for c in C], hq, hkv, T
        self.slot_in = np.arange(R, dtype=np.int32) if slot_in is None else np.asarray(slot_in, np.int32)
        self.slot_out = np.arange(R, 2 * R, dtype=np.int32) if slot_out is None else np.asarray(slot_out, np.int32)
        self.qkv = torch.randn((T + 1, hq + 2 * hkv, 128), generator=gen, device=DEV).to(torch.bfloat16)
        self.q, self.k, self.v = self.qkv[:, :hq], self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:]
        self.states = torch.randn((num_slots or 2 * R, hq, 128, 128), generator=gen, device=DEV) * 3
        self.log_decay = slopes(hq) if log_decay is None else np.asarray(log_decay, np.float32)
        self.batch = s2l.Batch([0] * R if P is None else P, C, np.zeros((R, 1), np.int32))
        to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
        self.state = s2l.LinearState(self.states, to(self.log_decay), to(self.slot_in), to(self.slot_out))
        self.out = torch.full((T + 2, hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)

    def run(self, stream=None):
        n = s2l.s2l_linear_attn_workspace_bytes(self.batch, self.hq)
        self.ws = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
        s2l.s2l_linear_attn(self.state, self.batch, self.q, self.k, self.v, SCALE, self.out, self.ws, stream)

    def check(self, requests=None, before=None):
        """Outputs and stored states against the oracle's, from the states `before` the call."""
        before = self.before if before is None else before
        q, k, v, out = (bf16_to_f64(t[:self.T]) for t in (self.q, self.k, self.v, self.out))
        cu = np.concatenate([[0], np.cumsum(self.C)])
        for r in range(len(self.C)) if requests is None else requests:
            a, b, C = cu[r], cu[r + 1], self.C[r]
            S0 = before[self.slot_in[r]].double().cpu().numpy() if self.slot_in[r] >= 0 else np.zeros((self.hq, 128, 128))
            o, S, A, B = linear_attn(q[a:b], k[a:b], v[a:b], self.log_decay, SCALE, S0)
            err, bound = np.abs(out[a:b] - o), 2.0 ** -8 * np.abs(o) + (2.0 ** -15 + (2 * C + 160) * 2.0 ** -24) * A
            assert np.all(err <= bound), (r, "out", np.argwhere(~(err <= bound))[:4], err.max())
            if C:
                assert np.linalg.norm(out[a:b] - o) <= 2.5e-3 * np.linalg.norm(o)
            if self.slot_out[r] >= 0:
                got = self.states[self.slot_out[r]].double().cpu().numpy()
                err, bound = np.abs(got - S), (2 * C + 16) * 2.0 ** -24 * B
                assert np.all(err <= bound), (r, "state", np.argwhere(~(err <= bound))[:4], err.max())
                assert np.linalg.norm(got - S) <= 2e-6 * np.linalg.norm(S)

    def run_and_check(self, requests=None):
        self.before = self.states.clone()
        self.run()
        torch.cuda.synchronize()
        self.check(requests)
        assert bool((self.out[self.T:] == 7).all())
        kept = np.setdiff1d(np.arange(self.states.shape[0]), self.slot_out)
        assert same(self.states[kept], self.before[kept])


@pytest.mark.parametrize("C,hq,hkv", [
    ([1], 32, 32), ([1], 1, 1), ([1] * 9, 8, 2), ([2, 0, 5, 1], 4, 4), ([3, 4, 15, 16, 17], 6, 2),
    ([31, 32, 33], 2, 2), ([63, 64, 65, 1], 3, 1), ([127, 0, 130], 2, 1), ([512], 4, 4), ([1000, 3, 257], 2, 2),
    ([2049], 2, 2), ([700, 1, 1, 1, 90, 4], 8, 1),
])
def test_equals_the_recurrence(C, hq, hkv):
    print(f"[linear] {C} {hq}/{hkv}", flush=True)
    Step(C, hq, hkv, seed=len(C) + hq).run_and_check()


def test_a_long_prompt():
    s = Step([8200], 2, 1, seed=50, slot_in=[-1], slot_out=[0], num_slots=1)
    s.run_and_check()


@pytest.mark.parametrize("C", [[1, 3, 0, 40], [600, 1, 70, 0]])
def test_slots(C):
    """Zero states, states that are not kept, snapshots and states advanced in place; other slots stay."""
    s = Step(C, 4, 2, seed=11, slot_in=[-1, 3, 5, 6], slot_out=[2, -1, 5, 0], num_slots=8)
    s.run_and_check()
    t = Step(C, 4, 2, seed=12, slot_in=[4, 1, -1, 3], slot_out=[4, 1, 7, 3], num_slots=8)
    t.run_and_check()


@pytest.mark.parametrize("C", [[2, 5, 1], [70, 40, 9], [600, 900, 33]])
def test_continuations_of_one_state(C):
    """Requests that all go on from the same slot, one of them without keeping what it makes of it."""
    Step(C, 4, 2, seed=30, slot_in=[1, 1, 1], slot_out=[0, -1, 2], num_slots=3).run_and_check()


@pytest.mark.parametrize("C", [[5, 2], [300, 70]])
def test_slots_out_of_range(C):
    """A bad slot to read makes NaN of the request; a bad slot to write stores nothing; others are as ever."""
    s = Step(C, 2, 2, seed=13, slot_in=[0, 1], slot_out=[2, 3], num_slots=4)
    s.before = s.states.clone()
    for bad_in, bad_out in (([4, 1], [2, 3]), ([-2, 1], [2, 3]), ([0, 1], [4, 3]), ([0, 1], [-5, 3])):
        s.states.copy_(s.before)
        s.state.slot_in.copy_(torch.tensor(bad_in, dtype=torch.int32))
        s.state.slot_out.copy_(torch.tensor(bad_out, dtype=torch.int32))
        s.run()
        torch.cuda.synchronize()
        s.check([1])
        if bad_in[0] != 0:
            assert bool(torch.isnan(s.out[:C[0]]).all()) and bool(torch.isnan(s.states[2]).all())
            assert same(s.states[:2], s.before[:2])
        else:
            s.slot_out = np.array([-1, 3])
            s.check()
            s.slot_out = np.array([2, 3])
            assert same(s.states[:3], s.before[:3])


@pytest.mark.parametrize("C", [[4], [200]])
def test_decays_at_their_ends(C):
    """No decay, decays that forget within a token, none at all left, and values above 0 (taken as 0)."""
    log_decay = [0.0, -1e-6, -0.5, -30.0, -200.0, -1e30, -np.inf, 0.25]
    s = Step(C, 8, 8, seed=14, log_decay=log_decay)
    s.run_and_check()
    assert bool(torch.isfinite(s.states).all())


@pytest.mark.parametrize("cut", [[1] * 20, [7, 13], [64, 1, 135], [100, 100]])
def test_any_chunking_gives_the_same(cut):
    """A sequence in chunks, its state advanced in place, against the sequence at once."""
    n, hq = sum(cut), 2
    whole = Step([n], hq, hq, seed=15, slot_in=[-1], slot_out=[0], num_slots=1)
    whole.run_and_check()
    outs, at, states = [], 0, torch.zeros((1, hq, 128, 128), device=DEV)
    for i, c in enumerate(cut):
        part = Step([c], hq, hq, seed=16, slot_in=[-1 if i == 0 else 0], slot_out=[0], num_slots=1)
        part.q, part.k, part.v = (t[at:at + c] for t in (whole.q, whole.k, whole.v))
        part.state.states = states
        part.run()
        outs.append(part.out[:c])
        at += c
    torch.cuda.synchronize()
    q, k, v = (bf16_to_f64(t[:n]) for t in (whole.q, whole.k, whole.v))
    o, S, A, B = linear_attn(q, k, v, whole.log_decay, SCALE, np.zeros((hq, 128, 128)))
    assert np.all(np.abs(bf16_to_f64(torch.cat(outs)) - o) <= 2.0 ** -8 * np.abs(o) + (2.0 ** -15 + (2 * n + 160) * 2.0 ** -24) * A)
    assert np.all(np.abs(states[0].double().cpu().numpy() - S) <= (2 * n + 16 * len(cut)) * 2.0 ** -24 * B)


@pytest.mark.parametrize("C,bad", [([9], 4), ([100], 37), ([100], 63), ([700], 640)])
def test_what_is_not_finite_reaches_no_row_before_it(C, bad):
    s = Step(C, 2, 2, seed=17)
    s.run()
    torch.cuda.synchronize()
    clean = s.out.clone()
    for t, value in ((s.v, float("nan")), (s.v, float("inf")), (s.k, float("nan")), (s.k, float("-inf"))):
        kept = t[bad, 1, 70].clone()
        t[bad, 1, 70] = value
        s.out.fill_(7.0)
        s.run()
        torch.cuda.synchronize()
        assert same(s.out[:bad], clean[:bad]) and same(s.out[:, 0], clean[:, 0])
        later = s.out[bad:s.T, 1]
        assert not bool(torch.isfinite(later[:, 70] if t is s.v else later).any())
        if t is s.v:
            rest = [c for c in range(128) if c != 70]
            assert same(later[:, rest], clean[bad:s.T, 1][:, rest])
        t[bad, 1, 70] = kept
    # a query reaches its own row alone
    s.q[bad, 0, 3] = float("nan")
    s.run()
    torch.cuda.synchronize()
    assert bool(torch.isnan(s.out[bad, 0]).all())
    s.out[bad, 0] = clean[bad, 0]
    assert same(s.out, clean)


def test_rows_behind_a_chunk_are_not_read():
    """A request's tail does not see the rows that follow it: the next request's, or none at all."""
    s = Step([45, 33], 2, 2, seed=18)
    s.qkv[s.T:] = float("nan")
    s.qkv[45:s.T] = float("nan")
    s.before = s.states.clone()
    s.run()
    torch.cuda.synchronize()
    s.check([0])


@pytest.mark.parametrize("C", [[3], [150, 900]])
def test_rows_at_odd_addresses(C):
    a = Step(C, 4, 2, seed=19)
    a.run()
    b = Step(C, 4, 2, seed=19)
    odd = lambda t: torch.zeros((t.shape[0], t.shape[1] * 128 + 3), dtype=torch.bfloat16, device=DEV)[:, 1:1 + t.shape[1] * 128].unflatten(1, (t.shape[1], 128))  # noqa: E731
    b.q, b.k, b.v, b.out = (odd(t).copy_(t) for t in (b.q, b.k, b.v, b.out))
    b.run()
    torch.cuda.synchronize()
    assert same(a.out, b.out) and same(a.states, b.states)


def test_states_past_four_gib():
    hq, slots = 64, 1100          # 4 MiB a slot
    for C in ([2, 1], [80, 40]):
        s = Step(C, hq, 8, seed=20, slot_in=[1, 0], slot_out=[2, 3], num_slots=4)
        s.run()
        big = torch.empty((slots, hq, 128, 128), device=DEV)
        gen = torch.Generator(device=DEV).manual_seed(20)
        t = Step(C, hq, 8, seed=20, slot_in=[1050, 0], slot_out=[1099, 1098], num_slots=4)
        big[1050], big[0] = s.states[1], s.states[0]
        t.state.states = big
        t.run()
        torch.cuda.synchronize()
        assert same(s.out, t.out) and same(s.states[2], big[1099]) and same(s.states[3], big[1098])
        del big, gen


@pytest.mark.parametrize("C", [[1, 1], [40, 1, 700]])
def test_graph_replays_and_repeats_are_the_same(C):
    s = Step(C, 4, 4, seed=21)
    s.run()
    torch.cuda.synchronize()
    ref = [s.out.clone(), s.states.clone()]
    stream, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(g, stream=stream):
            s2l.s2l_linear_attn(s.state, s.batch, s.q, s.k, s.v, SCALE, s.out, s.ws, stream)
    R = len(C)
    for _ in range(3):
        s.out.fill_(7.0)
        s.states[R:] = 0
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            g.replay()
        torch.cuda.synchronize()
        assert same(s.out, ref[0]) and same(s.states, ref[1])


def test_a_hybrid_step():
    """One step of a model with both kinds of layers, as a serving program runs it: rotation into the pages
    and attention over them in one layer, rotation and linear attention in the other."""
    from oracle.attention import ref_batch_attn
    from oracle.paged_kv import bf16_bits_to_f32
    from tests.gpu_util import from_bf16
    gen = torch.Generator(device=DEV).manual_seed(22)
    P, C, hq, hkv = np.array([40, 0, 130]), np.array([70, 5, 1]), 8, 2
    T = int(C.sum())
    tables = np.random.default_rng(22).permutation(30).astype(np.int32).reshape(3, 10)
    inv = (10000.0 ** -(np.arange(64) / 64)).astype(np.float32)
    rope = s2l.Rope(torch.from_numpy(inv).to(DEV))
    cache = s2l.PagedKVCache(*(torch.zeros((30, hkv, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    batch = s2l.Batch(P, C, tables)
    normal = lambda *shape: torch.randn(shape, generator=gen, device=DEV).to(torch.bfloat16)  # noqa: E731
    # the cached tokens, appended by an earlier step
    first = s2l.Batch(np.zeros(3, np.int32), P, tables)
    s2l.s2l_rope_kv_append(cache, first, rope, None, None, normal(int(P.sum()), hkv, 128), normal(int(P.sum()), hkv, 128))
    qkv = normal(T, hq + 2 * hkv, 128)
    q, out, lse = torch.empty((T, hq, 128), dtype=torch.bfloat16, device=DEV), torch.empty((T, hq, 128), dtype=torch.bfloat16, device=DEV), torch.empty((T, hq), device=DEV)
    s2l.s2l_rope_kv_append(cache, batch, rope, qkv[:, :hq], q, qkv[:, hq:hq + hkv], qkv[:, hq + hkv:])
    ws = torch.empty(s2l.s2l_attn_workspace_bytes(batch, hq, hkv), dtype=torch.uint8, device=DEV)
    plan = s2l.s2l_attn_plan(batch, hq, hkv, ws)
    s2l.s2l_chunk_prefill_attn(cache, batch, q, hq, SCALE, out, lse, plan, ws)
    # the linear layer goes on from its own projection of the attention's output
    lin = Step(C, hq, hkv, seed=23, slot_in=[0, -1, 2], slot_out=[0, 1, 2], num_slots=3, P=P)
    raw = lin.qkv.clone()
    s2l.s2l_rope_qk(batch, rope, lin.q, lin.q, lin.k, lin.k)
    lin.run_and_check()
    torch.cuda.synchronize()
    assert not same(raw, lin.qkv)
    o_ref = ref_batch_attn(bf16_bits_to_f32(from_bf16(q)).astype(np.float64), from_bf16(cache.k_pages), from_bf16(cache.v_pages),
                           tables, P.astype(np.int32), C.astype(np.int32), np.concatenate([[0], np.cumsum(C)]).astype(np.int32), hq, SCALE)[0]
    assert float(np.abs(bf16_to_f64(out) - o_ref).max()) <= 2e-2


@pytest.mark.parametrize("hq,hkv", [(32, 4), (6, 3)])
def test_many_requests(hq, hkv):
    """More requests than one search step holds, whole and cut, short and empty ones among them."""
    rng = np.random.default_rng(24)
    C = np.concatenate([rng.integers(0, 8, 60), rng.integers(6, 300, 70), [700, 0, 5, 6]])
    rng.shuffle(C)
    long = int(np.argmax(C))
    Step(C, hq, hkv, seed=24).run_and_check([0, 1, 63, 64, 65, 127, 128, 133, long])


def test_whole_chunks_of_many_heads():
    """Enough workgroups that no chunk is cut: states in place, with and without one to begin with."""
    C = [200, 64, 129, 31, 200, 96, 200, 7, 200, 200, 161, 33]
    s = Step(C, 64, 8, seed=25, slot_in=[0, -1, 2, 3, 4, 5, 6, -1, 8, 9, 10, 11], slot_out=list(range(12)), num_slots=12)
    assert s2l.s2l_linear_attn_workspace_bytes(s.batch, 64) == 0
    s.run_and_check([0, 1, 3, 7, 11])


@pytest.mark.parametrize("R,hq,hkv", [(2, 4, 2), (5, 8, 8), (70, 64, 8)])
def test_whole_chunks_few_and_many(R, hq, hkv):
    """Chunks in one launch, from workgroups that wait for CUs down to less than one for each: the outputs, the same
    at odd addresses, and values that are not finite."""
    C = [6 + (37 * r) % 91 for r in range(R)]
    a, b = (Step(C, hq, hkv, seed=29, slot_in=[-1] + list(range(1, R)), slot_out=list(range(R)), num_slots=R) for _ in range(2))
    assert s2l.s2l_linear_attn_workspace_bytes(a.batch, hq) == 0
    a.run_and_check([0, 1, R - 1])
    odd = torch.zeros((a.T + 1, (hq + 2 * hkv) * 128 + 3), dtype=torch.bfloat16, device=DEV)[:, 1:-2].unflatten(1, (hq + 2 * hkv, 128))
    odd.copy_(b.qkv)
    b.q, b.k, b.v = odd[:, :hq], odd[:, hq:hq + hkv], odd[:, hq + hkv:]
    b.run()
    torch.cuda.synchronize()
    assert same(a.out, b.out) and same(a.states, b.states)
    states, clean, bad = a.before, a.out.clone(), C[0] + 33     # in the second block of request 1
    for values in (a.q, b.q), (a.v, b.v):
        for s, t in zip((a, b), values):
            kept = t[bad, 1, 70].clone()
            t[bad, 1, 70] = float("inf")
            s.states.copy_(states)
            s.run()
            torch.cuda.synchronize()
            wrong = ~torch.isfinite(s.out[:s.T].float())
            if t is s.q:        # a query reaches its own row of its head
                assert bool(wrong[bad, 1].all()) and int(wrong.sum()) == 128
            else:               # a value its column of the rows from its own on, in all heads that share it
                rows, heads = slice(bad, C[0] + C[1]), slice(hq // hkv, 2 * hq // hkv)
                assert bool(wrong[rows, heads, 70].all()) and int(wrong.sum()) == (C[0] + C[1] - bad) * (hq // hkv)
            assert torch.equal(s.out[:s.T][~wrong], clean[:s.T][~wrong])
            t[bad, 1, 70] = kept


def test_rows_shared_and_far_apart():
    """A key row for all tokens (stride 0), and rows further apart than the fast copies take."""
    for C in ([3], [70], [300]):
        s = Step(C, 2, 2, seed=26)
        s.k = s.k[:1].expand(s.T, 2, 128)
        s.run_and_check()
    s = Step([9], 2, 2, seed=27)
    far = torch.empty(9 * ((1 << 24) + 8), dtype=torch.bfloat16, device=DEV).view(9, -1)[:, :256].unflatten(1, (2, 128))
    s.q = far.copy_(s.q[:9])
    s.run_and_check()


def test_workspace():
    s = Step([900, 40], 2, 2, seed=28)
    need = s2l.s2l_linear_attn_workspace_bytes(s.batch, 2)
    assert need > 0
    before = [s.states.clone(), s.out.clone()]
    for ws in (None, torch.empty(need - 1, dtype=torch.uint8, device=DEV)):
        with pytest.raises(s2l.S2LError) as e:
            s2l.s2l_linear_attn(s.state, s.batch, s.q, s.k, s.v, SCALE, s.out, ws)
        assert e.value.status == -3
    odd = torch.empty(need + 32, dtype=torch.uint8, device=DEV)[4:]
    with pytest.raises(s2l.S2LError) as e:
        s2l.s2l_linear_attn(s.state, s.batch, s.q, s.k, s.v, SCALE, s.out, odd)
    assert e.value.status == -1
    torch.cuda.synchronize()
    assert same(s.states, before[0]) and same(s.out, before[1])
    # nothing is expected of what a workspace holds, and nothing past its end is written
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
    s.before = before[0]
    s2l.s2l_linear_attn(s.state, s.batch, s.q, s.k, s.v, SCALE, s.out, ws)
    torch.cuda.synchronize()
    s.check()
    assert bool((ws[need:] == 0xFF).all())


def test_an_empty_batch():
    s = Step([0, 0], 2, 1, seed=29, slot_in=[1, -1], slot_out=[2, 3], num_slots=4)
    s.run_and_check()
    none = s2l.Batch([], [], np.zeros((0, 1), np.int32))
    empty = torch.zeros(0, dtype=torch.int32, device=DEV)
    rows = torch.zeros((0, 2, 128), dtype=torch.bfloat16, device=DEV)
    assert s2l.s2l_linear_attn_workspace_bytes(none, 2) == 0
    s2l.s2l_linear_attn(s2l.LinearState(s.states, s.state.log_decay, empty, empty), none, rows, rows, rows, SCALE, rows)
    rope = s2l.Rope(torch.ones(64, device=DEV))
    s2l.s2l_rope_qk(none, rope, rows, rows)
    cache = s2l.PagedKVCache(*(torch.zeros((1, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    s2l.s2l_rope_kv_append(cache, none, rope, None, None, rows, rows)
    torch.cuda.synchronize()
    assert not bool(cache.k_pages.any())


def test_two_streams_at_once():
    """Two batches on two streams, each with its own workspace, give what they give alone."""
    a, b = Step([700, 3], 4, 4, seed=30), Step([90, 1200, 1], 4, 2, seed=31)
    for s in (a, b):
        s.run()
        torch.cuda.synchronize()
        s.alone = [s.out.clone(), s.states.clone()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, stream in zip((a, b), streams):
            s2l.s2l_linear_attn(s.state, s.batch, s.q, s.k, s.v, SCALE, s.out, s.ws, stream)
    torch.cuda.synchronize()
    for s in (a, b):
        assert same(s.out, s.alone[0]) and same(s.states, s.alone[1])
