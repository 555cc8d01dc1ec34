"""Rotary positions in float64, written from the definition: pair i of a head turns by the angle
position * inv_freq[i], position that of the pair's axis."""
import numpy as np


def positions_of(prefix_lens, chunk_lens):
    """Position of every row of a varlen batch: P_r + i for row i of request r."""
    return np.concatenate([[]] + [np.arange(p, p + c) for p, c in zip(prefix_lens, chunk_lens)]).astype(np.int64)


def rotate(x, positions, inv_freq, pair_axes, adjacent=False, scale=1.0):
    """x [T][H][D] rotated; positions [axes][T].  Returns (y, reach): reach = |a| + |b| of each
    rotated element's pair times scale (0 where dims pass through), what errors of the sine and
    cosine act on."""
    x = np.asarray(x, np.float64)
    y, reach = x.copy(), np.zeros_like(x)
    pairs = len(inv_freq)
    for i in range(pairs):
        angle = np.asarray(positions[pair_axes[i]], np.float64) * np.float64(inv_freq[i])
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + pairs)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        y[:, :, a] = scale * (x[:, :, a] * c - x[:, :, b] * s)
        y[:, :, b] = scale * (x[:, :, b] * c + x[:, :, a] * s)
        reach[:, :, a] = reach[:, :, b] = scale * (np.abs(x[:, :, a]) + np.abs(x[:, :, b]))
    return y, reach
