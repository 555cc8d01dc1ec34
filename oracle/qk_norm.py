"""The norm of queries and keys for each head in float64: x / sqrt(mean x^2 + eps) * (weight + offset)."""
import numpy as np


def norm_heads(x, weight, eps, offset=0.0):
    """x [T][H][D]; weight [D] or None (no factor)."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).sum(-1, keepdims=True) / x.shape[-1] + np.float64(eps))
    return y if weight is None else y * (np.asarray(weight, np.float64) + np.float64(offset))
