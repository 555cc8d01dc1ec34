"""GPU: values near the end of the documented range of linear attention: a state of some 2^59 that is held up to 2^60 behind
its decay, read by queries whose sum over 128 dims is some 2^7.  Bounds as in test_gpu_linear."""
import numpy as np
import pytest
import torch

from oracle.linear_attn import linear_attn
from tests.gpu_util import bf16_to_f64
from tests.linear_forms import LONG
from tests.test_gpu_linear import SCALE, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["whole", "two", "pieces"])
def test_large_states(name):
    _, C, hq, hkv, _, _ = LONG[name]
    R = len(C)
    # 1.4 to 14 bits of decay a block: a fade comes after 4 to 41 of them
    s = Step(C, hq, hkv, seed=90, slot_in=list(range(R)), slot_out=list(range(R)), num_slots=R, log_decay=-np.geomspace(0.03, 0.3, hq))
    s.states.mul_(2.0 ** 57)
    s.v.mul_(2.0 ** 54)
    before = s.states.clone()
    s.run()
    torch.cuda.synchronize()
    heads, r = [0, 1, hq // 2, hq - 1], 0
    shared = [h // (hq // hkv) for h in heads]
    q, k, v, out = (bf16_to_f64(t[:C[r]][:, n]) for t, n in ((s.q, heads), (s.k, shared), (s.v, shared), (s.out, heads)))
    o, S, A, B = linear_attn(q, k, v, s.log_decay[heads], SCALE, before[r][heads].double().cpu().numpy())
    peak = max(np.abs(before[r][heads].double().cpu().numpy()).max(), B.max())
    assert 2.0 ** 59 < peak < 2.0 ** 67 and 2.0 ** 65 < A.max() / SCALE < 2.0 ** 67       # near its end, within the range
    assert np.all(np.abs(out - o) <= 2.0 ** -8 * np.abs(o) + (2.0 ** -15 + (2 * C[r] + 160) * 2.0 ** -24) * A)
    assert np.all(np.abs(s.states[r][heads].double().cpu().numpy() - S) <= (2 * C[r] + 16) * 2.0 ** -24 * B)
    assert bool(torch.isfinite(s.out[:s.T].float()).all()) and bool(torch.isfinite(s.states).all())
