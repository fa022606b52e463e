"""Oracle: attention over packed sequences (float64, plain NumPy).

TEST INFRASTRUCTURE ONLY -- see the package docstring.

Sequence i has the query rows q_offsets[i] : q_offsets[i + 1] of q [total_q, H, 128] and m_i key rows from
k_offsets[i] of k, v [total_k, Hk, 128]; head h reads key head h // (H // Hk).  Query t of n_i sees every prefix row
and its own keys c < m_i, if causal those with c <= t + m_i - n_i:

    O = sum_c softmax(sm_scale <q, k_c>) v_c,   lse = ln sum_c exp(sm_scale <q, k_c>)

A query that sees nothing gives O = 0 and lse = -inf.  Rows of no sequence are NaN in both.
"""

from __future__ import annotations

import numpy as np


def attention(q, k, v, q_offsets, k_offsets, sm_scale, causal, k_lens=None, prefix_k=None, prefix_v=None):
    """(O [total_q, H, 128], lse [H, total_q])."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    H, Hk = q.shape[1], k.shape[1]
    out = np.full(q.shape, np.nan)
    lse = np.full((H, q.shape[0]), np.nan)
    for i in range(len(q_offsets) - 1):
        q0, q1 = int(q_offsets[i]), int(q_offsets[i + 1])
        k0 = int(k_offsets[i])
        m = int(k_lens[i]) if k_lens is not None else int(k_offsets[i + 1]) - k0
        n = q1 - q0
        for h in range(H):
            g = h // (H // Hk)
            own_k, own_v = k[k0:k0 + m, g], v[k0:k0 + m, g]
            for t in range(n):
                seen = min(max(t + 1 + m - n, 0), m) if causal else m
                kk, vv = own_k[:seen], own_v[:seen]
                if prefix_k is not None:
                    kk = np.concatenate((np.asarray(prefix_k, dtype=np.float64)[:, g], kk))
                    vv = np.concatenate((np.asarray(prefix_v, dtype=np.float64)[:, g], vv))
                z = sm_scale * (kk @ q[q0 + t, h])
                top = z.max() if len(z) else -np.inf
                if top == -np.inf:
                    out[q0 + t, h], lse[h, q0 + t] = 0.0, -np.inf
                    continue
                e = np.exp(z - top)
                out[q0 + t, h] = e @ vv / e.sum()
                lse[h, q0 + t] = top + np.log(e.sum())
    return out, lse
