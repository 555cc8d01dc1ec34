"""GPU: states of long chunks that no cut shortens, against float64, by a bound that does not grow with the chunk.

A token joins the running state by two powers of the decay and stays in it under two more at most (of
what is older than one fade, less than 2^-28 is left).  A power is the hardware's exp2 (one ulp, 2^-23
of it) of an argument with two roundings of at most 2^-26 each (2^-25 in all); each of the four is multiplied in with a
rounding of 2^-24.  A block's sums round the state six times (three terms, halves of the block apart), and a
rounding b blocks before the end counts l^(32 b): independent ones add up to sqrt(6 / (1 - l^64)) 2^-24.
Tokens are independent, so all of that bounds the norm of the state's error as a part of its norm.
"""
import numpy as np
import pytest
import torch

from tests.gpu_util import bf16_to_f64
from tests.test_gpu_linear import Step

pytestmark = pytest.mark.gpu


def bound(log_decay):
    return 4 * (2.0 ** -23 + 2.0 ** -25) + 4 * 2.0 ** -24 + np.sqrt(6 / -np.expm1(64 * log_decay)) * 2.0 ** -24


# decays from half of a state kept over 140 tokens to half of it over one, and those between that lose most where a
# power's exponent is rounded whole
DECAYS = -np.concatenate([np.geomspace(0.005, 0.7, 60), [0.00711, 0.0156, 0.0229, 0.2224]])


@pytest.mark.parametrize("C", [[4205, 1494, 2049] * 3 + [4205] * 5, [2100, 2049], [1494, 1400]],
                         ids=["a workgroup a head", "two workgroups a head", "two workgroups a head, shorter"])
def test_states_of_long_whole_chunks(C):
    """Uncut chunks: the state is held up to 2^60 behind its decay."""
    R, hq, hkv = len(C), 64, 8
    s = Step(C, hq, hkv, seed=40, slot_in=[-1] + list(range(1, R)), slot_out=list(range(R)), num_slots=R, log_decay=DECAYS)
    before = s.states[:3].double().cpu().numpy()
    s.run()
    torch.cuda.synchronize()
    assert s.ws is None        # not cut
    cu, g, worst = np.concatenate([[0], np.cumsum(C)]), s.log_decay.astype(np.float64), []
    for r in range(min(R, 3)):
        k, v = (bf16_to_f64(t[cu[r]:cu[r + 1]]) for t in (s.k, s.v))
        left = np.arange(C[r] - 1, -1, -1)
        for h in range(hq):
            S = (k[:, h // 8] * np.exp(g[h] * left)[:, None]).T @ v[:, h // 8]
            if r > 0:
                S += np.exp(g[h] * C[r]) * before[r, h]
            err = np.linalg.norm(s.states[r, h].double().cpu().numpy() - S) / np.linalg.norm(S)
            worst.append((err / bound(g[h]), err, r, h))
    print(f"[precision] {C[:3]}: largest {max(worst)}, mean {np.mean([w[1] for w in worst]):.2e}", flush=True)
    assert max(worst)[0] <= 1, sorted(worst)[-4:]
