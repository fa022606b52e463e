"""The oracles of Q / K norm and rotation and of packed attention, against closed forms and the dense oracle."""

import math

import numpy as np
import pytest

from oracle import attention as oa
from oracle import packed, rotary

FREQS = [10000.0 ** (-i / n) for n in (22, 21, 21) for i in range(n)]
PAIRS = (22, 21, 21)


def test_norm_of_a_head_and_of_a_token():
    x = np.zeros((1, 1, 2, 128))
    x[0, 0, 0], x[0, 0, 1] = 3.0, 4.0
    w = np.full(128, 2.0)
    assert np.allclose(rotary.norm(x, "head", w, 0.0), 2.0)
    y = rotary.norm(x, "token", np.stack([w, w]), 0.0)
    rms = math.sqrt((9 + 16) / 2)
    assert np.allclose(y[0, 0, 0], 6 / rms) and np.allclose(y[0, 0, 1], 8 / rms)
    assert np.allclose(rotary.norm(x * 0, "head", w, 1e-6), 0.0)


@pytest.mark.parametrize("adjacent", [True, False])
def test_rotation_is_a_turn_by_position(rng, adjacent):
    x = rng.standard_normal((1, 1, 1, 128))
    at = rotary.rotate(x, np.array([[0], [0], [0]]), PAIRS, FREQS, adjacent)
    assert np.allclose(at, x)
    # (1, 0) at position p turns to (cos, sin)
    e = np.zeros((1, 1, 1, 128))
    i, j = (2 * 30, 2 * 30 + 1) if adjacent else (30, 94)     # pair 30 lies on axis 1
    e[..., i] = 1
    y = rotary.rotate(e, np.array([[5], [7], [9]]), PAIRS, FREQS, adjacent)
    assert np.isclose(y[0, 0, 0, i], math.cos(7 * FREQS[30])) and np.isclose(y[0, 0, 0, j], math.sin(7 * FREQS[30]))
    assert np.isclose((y ** 2).sum(), 1)


def test_rotated_products_depend_on_the_difference_of_positions(rng):
    q, k = rng.standard_normal((2, 1, 1, 1, 128))

    def dot(p, r):
        f = [rotary.rotate(x, np.full((3, 1), n), PAIRS, FREQS, True) for x, n in ((q, p), (k, r))]
        return float((f[0] * f[1]).sum())

    assert np.isclose(dot(12, 3), dot(109, 100)) and not np.isclose(dot(12, 3), dot(13, 3))


def test_one_sequence_equals_the_dense_oracle(rng):
    q, k, v = rng.standard_normal((3, 70, 2, 128))
    O, lse = packed.attention(q, k, v, [0, 70], [0, 70], 0.1, False)
    rp, ci = np.arange(0, 9, 2), np.tile([0, 1], 4)
    D, dl = oa.attention(q[None], k[None], v[None], rp, ci, 0.1, 1)
    assert np.allclose(O, D[0]) and np.allclose(lse, dl[0])


def test_causal_rows_see_up_to_themselves(rng):
    q, k, v = rng.standard_normal((3, 9, 1, 128))
    O, lse = packed.attention(q, k, v, [0, 4, 9], [0, 4, 9], 0.1, True)
    assert np.allclose(O[0], v[0]) and np.allclose(O[4], v[4])
    part, _ = packed.attention(q[:3], k[:3], v[:3], [0, 3], [0, 3], 0.1, True)
    assert np.allclose(part, O[:3])
    # more queries than keys: the first see nothing
    O, lse = packed.attention(q, k, v, [0, 4], [0, 2], 0.1, True)
    assert (O[:2] == 0).all() and np.isneginf(lse[0, :2]).all() and np.allclose(O[2], v[0])
    assert np.isnan(O[4:]).all()


def test_a_prefix_is_keys_ahead_of_every_sequence(rng):
    q, k, v = rng.standard_normal((3, 6, 4, 128))
    pk, pv = rng.standard_normal((2, 5, 2, 128))
    O, _ = packed.attention(q, k[:, :2], v[:, :2], [0, 2, 6], [0, 2, 6], 0.1, True, prefix_k=pk, prefix_v=pv)
    for a, b in ((0, 2), (2, 6)):
        kk, vv = np.concatenate((pk, k[a:b, :2])), np.concatenate((pv, v[a:b, :2]))
        R, _ = packed.attention(q[a:b], kk, vv, [0, b - a], [0, len(kk)], 0.1, True)
        assert np.allclose(O[a:b], R)
