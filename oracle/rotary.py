"""Oracle: norm and rotation of Q and K (float64, plain NumPy).

TEST INFRASTRUCTURE ONLY -- see the package docstring.

For a tensor x [B, S, H, 128] and each token:

    y = x / sqrt(mean(x^2) + eps) * w      mean over a head (w [128]) or over the token's heads (w [H, 128])
    (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = position on the pair's axis * freqs[p]

for the pairs p = 0 .. 63 of a head, the values (2p, 2p + 1) or (p, p + 64), dealt to the axes in order.
"""

from __future__ import annotations

import numpy as np


def norm(x, kind, weight, eps):
    x = np.asarray(x, dtype=np.float64)
    if kind is None:
        return x
    over = -1 if kind == "head" else (-2, -1)
    w = np.asarray(weight, dtype=np.float64)
    if kind == "token":
        w = w.reshape(x.shape[-2:])
    return x / np.sqrt((x * x).mean(axis=over, keepdims=True) + eps) * w


def rotate(x, positions, pairs, freqs, adjacent):
    """positions int [axes, S] or [axes, B, S]."""
    x = np.asarray(x, dtype=np.float64)
    pos = np.asarray(positions, dtype=np.float64)
    if pos.ndim == 2:
        pos = np.broadcast_to(pos[:, None], (pos.shape[0], x.shape[0], pos.shape[1]))
    out = np.empty_like(x)
    p = 0
    for axis, count in enumerate(pairs):
        for _ in range(count):
            t = (pos[axis] * freqs[p])[:, :, None]
            i, j = (2 * p, 2 * p + 1) if adjacent else (p, p + 64)
            a, b = x[..., i], x[..., j]
            out[..., i] = a * np.cos(t) - b * np.sin(t)
            out[..., j] = a * np.sin(t) + b * np.cos(t)
            p += 1
    return out


def norm_rotate(x, kind=None, weight=None, eps=1e-6, positions=None, pairs=None, freqs=None, adjacent=True):
    y = norm(x, kind, weight, eps)
    return y if positions is None else rotate(y, positions, pairs, freqs, adjacent)
