"""The oracles of rotary positions and linear attention against properties and brute force (CPU)."""
import numpy as np
import pytest

from oracle.linear_attn import linear_attn
from oracle.rotary import positions_of, rotate


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_is_a_complex_product(adjacent):
    rng = np.random.default_rng(0)
    x, pos, inv = rng.normal(size=(5, 3, 20)), rng.integers(-50, 10 ** 6, (2, 5)), rng.random(8)
    axes = [0, 1, 1, 0, 1, 0, 0, 1]
    y, reach = rotate(x, pos, inv, axes, adjacent, 0.7)
    assert np.array_equal(y[..., 16:], x[..., 16:]) and not reach[..., 16:].any()
    split = lambda t: t[..., 0:16:2] + 1j * t[..., 1:16:2] if adjacent else t[..., :8] + 1j * t[..., 8:16]  # noqa: E731
    turn = np.exp(1j * pos[axes].T * inv)[:, None]
    assert np.allclose(split(y), 0.7 * split(x) * turn, rtol=0, atol=1e-9)


def test_scores_see_relative_positions_only():
    rng = np.random.default_rng(1)
    q, k, inv = rng.normal(size=(1, 1, 128)), rng.normal(size=(1, 1, 128)), 10000.0 ** -(np.arange(64) / 64)
    score = lambda m, n: float(np.sum(rotate(q, [[m]], inv, [0] * 64)[0] * rotate(k, [[n]], inv, [0] * 64)[0]))  # noqa: E731
    assert abs(score(7, 3) - score(1007, 1003)) < 1e-9 and abs(score(7, 3) - score(7, 4)) > 1e-6


def test_positions_of_a_batch():
    assert positions_of([5, 0, 9], [2, 0, 3]).tolist() == [5, 6, 9, 10, 11]


def test_linear_attention_is_the_decayed_sum():
    """out_i = scale sum_j l^(i-j) (q_i . k_j) v_j + scale l^(i+1) q_i S0, heads shared in groups."""
    rng = np.random.default_rng(2)
    C, hq, hkv, D = 9, 4, 2, 6
    q, k, v = rng.normal(size=(C, hq, D)), rng.normal(size=(C, hkv, D)), rng.normal(size=(C, hkv, D))
    S0, g = rng.normal(size=(hq, D, D)), np.array([-0.5, 0.0, -3.0, 0.3])
    out, S, A, B = linear_attn(q, k, v, g, 0.25, S0)
    for h in range(hq):
        lam, kh, vh = np.exp(min(g[h], 0.0)), k[:, h // 2], v[:, h // 2]
        for i in range(C):
            o = sum(lam ** (i - j) * (q[i, h] @ kh[j]) * vh[j] for j in range(i + 1)) + lam ** (i + 1) * (q[i, h] @ S0[h])
            assert np.allclose(out[i, h], 0.25 * o, atol=1e-12)
        end = lam ** C * S0[h] + sum(lam ** (C - 1 - j) * np.outer(kh[j], vh[j]) for j in range(C))
        assert np.allclose(S[h], end, atol=1e-12)
    assert np.all(A >= np.abs(out) - 1e-12) and np.all(B >= np.abs(S) - 1e-12)


@pytest.mark.parametrize("cut", [1, 4, 8])
def test_linear_attention_in_two_chunks(cut):
    rng = np.random.default_rng(3)
    q, k, v = (rng.normal(size=(9, 2, 5)) for _ in range(3))
    g, S0 = [-0.1, -0.7], np.zeros((2, 5, 5))
    out, S = linear_attn(q, k, v, g, 1.0, S0)[:2]
    o1, S1 = linear_attn(q[:cut], k[:cut], v[:cut], g, 1.0, S0)[:2]
    o2, S2 = linear_attn(q[cut:], k[cut:], v[cut:], g, 1.0, S1)[:2]
    assert np.allclose(np.concatenate([o1, o2]), out, atol=1e-12) and np.allclose(S2, S, atol=1e-12)
    empty = linear_attn(q[:0], k[:0], v[:0], g, 1.0, S1)
    assert np.array_equal(empty[1], S1)
