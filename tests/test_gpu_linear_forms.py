"""GPU: each form of linear attention over enough blocks that its ring of tiles goes round several times, with tiles
copied straight into LDS and through registers (rows at odd addresses).  Bounds as in test_gpu_linear."""
import numpy as np
import pytest
import torch

from oracle.linear_attn import linear_attn
from tests.gpu_util import DEV, bf16_to_f64
from tests.linear_forms import CUT, LONG
from tests.test_gpu_linear import SCALE, Step, same

pytestmark = pytest.mark.gpu


def check_heads(s, before, heads, requests):
    """As Step.check, of some heads."""
    cu, shared = np.concatenate([[0], np.cumsum(s.C)]), [h // (s.hq // s.hkv) for h in heads]
    for r in requests:
        rows, C = slice(cu[r], cu[r + 1]), s.C[r]
        q, k, v, out = (bf16_to_f64(t[rows][:, n]) for t, n in ((s.q, heads), (s.k, shared), (s.v, shared), (s.out, heads)))
        S0 = before[s.slot_in[r]][heads].double().cpu().numpy() if s.slot_in[r] >= 0 else np.zeros((len(heads), 128, 128))
        o, S, A, B = linear_attn(q, k, v, s.log_decay[heads], SCALE, S0)
        assert np.all(np.abs(out - o) <= 2.0 ** -8 * np.abs(o) + (2.0 ** -15 + (2 * C + 160) * 2.0 ** -24) * A), (r, "out")
        assert np.linalg.norm(out - o) <= 2.5e-3 * np.linalg.norm(o), (r, "out")
        got = s.states[s.slot_out[r]][heads].double().cpu().numpy()
        assert np.all(np.abs(got - S) <= (2 * C + 16) * 2.0 ** -24 * B), (r, "state")
        assert np.linalg.norm(got - S) <= 2e-6 * np.linalg.norm(S), (r, "state")


def odd(t):
    """The same rows at odd addresses, a row's length apart that is no multiple of 16 bytes."""
    n = t.shape[1] * 128
    return torch.zeros((t.shape[0], n + 3), dtype=torch.bfloat16, device=DEV)[:, 1:1 + n].unflatten(1, (t.shape[1], 128)).copy_(t)


@pytest.mark.parametrize("name", LONG)
def test_many_blocks_in_each_form(name):
    form, C, hq, hkv, _, _ = LONG[name]
    R = len(C)
    print(f"[forms] {name}", flush=True)

    def make():
        return Step(C, hq, hkv, seed=60, slot_in=[-1] + list(range(1, R)), slot_out=list(range(R)), num_slots=R)
    s = make()
    before = s.states.clone()
    s.run()
    torch.cuda.synchronize()
    assert (s.ws is not None) == (form == CUT)
    check_heads(s, before, [0, hq // 2, hq - 1], range(R) if max(C) < 1000 else [0, R - 1])
    assert bool((s.out[s.T:] == 7).all())
    # rows that the copies into LDS do not take: K and V alone, Q alone, all of them
    for names in ("kv", "q", "qkv"):
        t = make()
        for n in names:
            setattr(t, n, odd(getattr(t, n)))
        t.run()
        torch.cuda.synchronize()
        assert same(s.out, t.out) and same(s.states, t.states), names


@pytest.mark.parametrize("name", LONG)
def test_many_blocks_replayed(name):
    """Captured, with rows at odd addresses: replays, with eager calls between them, give the same bits."""
    import paper_2604_16395_amd as s2l
    _, C, hq, hkv, _, _ = LONG[name]
    R = len(C)
    s = Step(C, hq, hkv, seed=61, slot_in=list(range(R)), slot_out=list(range(R, 2 * R)))
    s.v = odd(s.v)
    s.run()
    torch.cuda.synchronize()
    ref = [s.out.clone(), s.states.clone()]
    stream, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream), torch.cuda.graph(g, stream=stream):
        s2l.s2l_linear_attn(s.state, s.batch, s.q, s.k, s.v, SCALE, s.out, s.ws, stream)
    for replay in (True, False, True, True):
        s.out.fill_(7.0)
        s.states[R:] = 0
        torch.cuda.synchronize()
        if replay:
            with torch.cuda.stream(stream):
                g.replay()
        else:
            s.run()
        torch.cuda.synchronize()
        assert same(s.out, ref[0]) and same(s.states, ref[1])
