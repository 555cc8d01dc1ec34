"""Linear attention with a decay for each head, in float64, token after token:
S <- l S + k v^T, out = scale q S, l = exp(log_decay)."""
import numpy as np


def linear_attn(q, k, v, log_decay, scale, state):
    """One request: q [C][Hq][D], k and v [C][Hkv][D], state [Hq][D][D] (k, v).  Returns (out, state
    after the chunk, A, B): A and B are out and the state with every product's absolute value."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    hq, hkv = q.shape[1], k.shape[1]
    head = np.arange(hq) // (hq // hkv)
    decay = np.exp(np.minimum(np.asarray(log_decay, np.float64), 0.0))[:, None, None]
    S, B = np.array(state, np.float64), np.abs(np.asarray(state, np.float64))
    out, A = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(q.shape[0]):
        kv = k[i, head][:, :, None] * v[i, head][:, None, :]
        S = decay * S + kv
        B = decay * B + np.abs(kv)
        out[i] = scale * np.einsum("hk,hkv->hv", q[i], S)
        A[i] = abs(scale) * np.einsum("hk,hkv->hv", np.abs(q[i]), B)
    return out, S, A, B
