"""GPU: a layer's step with the operators together, as a serving program runs it: rows of one projection normed,
rotated and quantised into MXFP4 pages, attention over them, and the chunk read back; chunk after chunk, decoded,
captured into graphs, and on streams of its own."""
import numpy as np
import pytest
import torch

import paper_2604_16395_amd as s2l
from oracle.attention import ref_chunk_attn_blocked
from tests.gpu_util import DEV, SCALE, bf16_to_f64

pytestmark = pytest.mark.gpu

HQ, HKV = 8, 2
INV = torch.from_numpy((10000.0 ** -(np.arange(64) / 64)).astype(np.float32))


class Layer:
    """One layer's cache, norm and rotation, and the rows of its requests' sequences."""

    def __init__(self, lengths, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.lengths = lengths
        self.rows = [torch.randn((n, HQ + 2 * HKV, 128), generator=gen, device=DEV).to(torch.bfloat16) for n in lengths]
        need = [-(-n // 16) for n in lengths]
        order = np.random.default_rng(seed).permutation(sum(need))
        self.tables = np.zeros((len(lengths), max(need)), np.int32)
        for r, n in enumerate(need):
            self.tables[r, :n] = order[sum(need[:r]):sum(need[:r + 1])]
        self.cache = s2l.PagedKVCache(*(torch.randint(0, 256, (sum(need), HKV, s2l.MXFP4_RUN_BYTES), dtype=torch.uint8, generator=gen, device=DEV)
                                        for _ in range(2)))
        self.norm = s2l.QKNorm(*(1 + 0.2 * torch.randn(128, generator=gen, device=DEV) for _ in range(2)))
        self.rope = s2l.Rope(INV.to(DEV))

    def buffers(self, P, C):
        """A step's batch, projected rows and buffers."""
        T = sum(C)
        b = dict(batch=s2l.Batch(P, C, self.tables), qkv=torch.cat([x[p:p + c] for x, p, c in zip(self.rows, P, C)]))
        b["ws"] = torch.empty(s2l.s2l_attn_workspace_bytes(b["batch"], HQ, HKV), dtype=torch.uint8, device=DEV)
        b["q"], b["out"] = (torch.zeros((T, HQ, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        b["k"], b["v"] = (torch.zeros((T, HKV, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return b

    def step(self, b, stream=None):
        batch, qkv = b["batch"], b["qkv"]
        s2l.s2l_norm_rope_kv_append(self.cache, batch, self.norm, self.rope, qkv[:, :HQ], b["q"], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], stream)
        plan = s2l.s2l_attn_plan(batch, HQ, HKV, b["ws"], stream=stream)
        s2l.s2l_chunk_prefill_attn(self.cache, batch, b["q"], HQ, SCALE, b["out"], None, plan, b["ws"], stream)
        s2l.s2l_kv_read(self.cache, batch, s2l.S2L_READ_CHUNK, batch.cu_chunk, b["k"], b["v"], stream)

    def check(self, r, q, k, v, out, P):
        """Rows of one request from position P on, over the values that were read back."""
        ref = ref_chunk_attn_blocked(*(bf16_to_f64(x) for x in (q, k, v)), P, SCALE, with_abs=True, spread=True)
        o, a, spread = ref[0], ref[2], ref[3]
        u = 2.0 ** -8
        err = np.abs(bf16_to_f64(out) - o)
        assert (err <= u * np.abs(o) + 2.02 * u * spread + 2.0 ** -16 * a + 1e-6).all(), (r, err.max())


def test_chunks_then_single_tokens():
    """Three requests advance by chunks that end inside pages, then by one token each; every row's output is the
    attention over all values read back so far."""
    layer = Layer([150, 77, 40], 1)
    done, k, v, q, out = [0, 0, 0], [[], [], []], [[], [], []], [[], [], []], [[], [], []]
    for C in ([100, 1, 0], [30, 70, 33], [1, 1, 1], [1, 0, 1], [4, 2, 1]):
        b = layer.buffers(done, C)
        layer.step(b)
        torch.cuda.synchronize()
        at = 0
        for r, c in enumerate(C):
            for to, name in ((k, "k"), (v, "v"), (q, "q"), (out, "out")):
                to[r].append(b[name][at:at + c])
            at += c
            done[r] += c
    for r in range(3):
        layer.check(r, torch.cat(q[r]), torch.cat(k[r]), torch.cat(v[r]), torch.cat(out[r]), 0)


def test_replayed_graphs_that_share_a_workspace():
    """Two captured steps, of a chunk and of single tokens, over one workspace: every replay, in turn, with eager work
    between, gives the eager step's bits."""
    layer = Layer([600, 90], 2)
    steps = [layer.buffers([500, 0], [80, 80]), layer.buffers([580, 80], [1, 1])]
    if steps[0]["ws"].numel() < steps[1]["ws"].numel():
        steps[0]["ws"] = steps[1]["ws"]
    steps[1]["ws"] = steps[0]["ws"]
    before = layer.buffers([0, 0], [500, 0])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer.step(before)
        want = []
        for b in steps:
            layer.step(b)
            want.append({n: b[n].clone() for n in ("q", "out", "k", "v")})
    torch.cuda.synchronize()
    graphs = []
    for b in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream), torch.cuda.graph(g, stream=stream):
            layer.step(b)
        graphs.append(g)
    torch.cuda.synchronize()
    for turn in range(3):
        for b, g, w in zip(steps, graphs, want):
            for n in w:
                b[n].zero_()
            junk = torch.randn(1 << 20, device=DEV).sum()
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                g.replay()
            torch.cuda.synchronize()
            assert torch.isfinite(junk)
            for n in w:
                assert torch.equal(b[n].view(torch.int16), w[n].view(torch.int16)), (turn, n)


def test_two_streams_at_once():
    """Two layers' steps in flight together on streams of their own, given by argument, give the bits they give alone."""
    layers = [Layer([700, 33], 3), Layer([64, 900], 4)]
    alone = []
    for layer in layers:
        b = layer.buffers([0, 0], [l - 1 for l in layer.lengths])
        layer.step(b)
        torch.cuda.synchronize()
        alone.append((b, {n: b[n].clone() for n in ("q", "out", "k", "v")}, layer.cache.k_pages.clone()))
    streams = [torch.cuda.Stream() for _ in layers]
    for turn in range(3):
        for layer, (b, _, _) in zip(layers, alone):
            for n in ("q", "out", "k", "v"):
                b[n].zero_()
        torch.cuda.synchronize()
        for layer, (b, _, _), stream in zip(layers, alone, streams):
            layer.step(b, stream)
        torch.cuda.synchronize()
        for layer, (b, w, pages) in zip(layers, alone):
            assert all(torch.equal(b[n].view(torch.int16), w[n].view(torch.int16)) for n in w) and torch.equal(layer.cache.k_pages, pages)


def test_a_batch_whose_requests_share_their_prefix():
    """Two requests over the same cached pages, one of them twice as long: rows of equal tokens give equal bits."""
    layer = Layer([200, 200], 5)
    layer.rows[1] = layer.rows[0]
    layer.tables[1, :4] = layer.tables[0, :4]
    first = layer.buffers([0, 0], [64, 0])
    layer.step(first)
    b = layer.buffers([64, 64], [50, 100])
    layer.step(b)
    torch.cuda.synchronize()
    assert torch.equal(b["k"][:50], b["k"][50:100]) and torch.equal(b["q"][:50], b["q"][50:100])
    layer.check(0, b["q"][:50], torch.cat([first["k"], b["k"][:50]]), torch.cat([first["v"], b["v"][:50]]), b["out"][:50], 64)
    layer.check(1, b["q"][50:], torch.cat([first["k"], b["k"][50:]]), torch.cat([first["v"], b["v"][50:]]), b["out"][50:], 64)
