"""The float64 definitions of the transformer-layer operators, pinned to scalar
loops, closed forms and invariants."""

import math

import numpy as np
import pytest

import oracle
from oracle import transformer as T


def _rng(seed):
    return np.random.default_rng(seed)


def test_row_codes_hand_values():
    c, top = T.row_codes([[0.0, 0.0], [2.0, -1.0], [254.0, 3.0], [1.0, np.nan]])
    assert top[:2].tolist() == [0.0, 2.0]
    # -127 / 2 is half-way between two codes and goes to the even one; 127 * 3 / 254 = 1.5 too
    assert c[:3].tolist() == [[0, 0], [127, -64], [127, 2]]


def test_qdense_against_integer_loops():
    r = _rng(1)
    x, w = r.normal(size=(5, 37)), r.normal(size=(4, 37))
    x[2] = 0
    y = T.qdense(x, w)
    for m in range(5):
        for n in range(4):
            ax, aw = max(abs(v) for v in x[m]), max(abs(v) for v in w[n])
            s = sum(int(round(127 * a / ax)) * int(round(127 * b / aw)) for a, b in zip(x[m], w[n])) if ax else 0
            assert y[m, n] == pytest.approx(s * ax * aw / 127 ** 2, rel=1e-14, abs=0)
    x[3, 5], x[4, 0] = np.inf, np.nan
    y2 = T.qdense(x, w)
    assert np.isnan(y2[3:]).all() and np.array_equal(y2[:3], y[:3])


def test_qdense_is_near_the_product():
    r = _rng(2)
    x, w = r.normal(size=(16, 512)), r.normal(size=(24, 512))
    y, ref = T.qdense(x, w), x @ w.T
    # each code is off by half a step at most; the sum of 512 such errors is far below its bound
    assert np.abs(y - ref).max() < 512 * (np.abs(x).max() * np.abs(w).max() / 127)
    assert np.linalg.norm(y - ref) < 0.02 * np.linalg.norm(ref)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_against_complex_numbers(interleaved):
    r = _rng(3)
    x = r.normal(size=(6, 2, 12))
    theta = np.array([1.0, 0.3, 0.01, 0.002])  # 8 of 12 columns turn
    pos = np.array([0, 1, -3, 77, 100000, 5])
    y = T.rotate(x, pos, theta, 1.25, interleaved)
    for m in range(6):
        for h in range(2):
            for i, t in enumerate(theta):
                a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + 4)
                z = complex(x[m, h, a], x[m, h, b]) * 1.25 * np.exp(1j * float(pos[m]) * t)
                assert abs(y[m, h, a] - z.real) < 1e-12 and abs(y[m, h, b] - z.imag) < 1e-12
    assert np.array_equal(y[..., 8:], x[..., 8:])
    assert np.allclose(y[0, :, :8], 1.25 * x[0, :, :8], rtol=1e-15)  # position 0 does not turn


def test_rotated_products_depend_on_the_distance():
    r = _rng(4)
    attrs = {"heads": 1, "kv_heads": 1, "head_dim": 16}
    q, k = r.normal(size=16), r.normal(size=16)

    def dot(i, j):
        y = T.rotary(attrs, np.array([np.concatenate([q, k])] * 2), [i, j])
        return y[0, :16] @ y[1, 16:]

    assert dot(5, 3) == pytest.approx(dot(1005, 1003), rel=1e-9)


def test_scaled_angles():
    a = {"heads": 1, "head_dim": 64, "base": 10000.0}
    plain, _ = T.rotary_theta(a)
    assert plain[0] == 1.0 and plain[-1] == pytest.approx(10000.0 ** (-62 / 64))
    lin, _ = T.rotary_theta(dict(a, scaling={"type": "linear", "factor": 4.0}))
    assert np.allclose(lin, plain / 4)
    ntk, _ = T.rotary_theta(dict(a, scaling={"type": "ntk", "factor": 4.0}))
    assert ntk[0] == 1.0 and ntk[-1] == pytest.approx(plain[-1] / 4, rel=1e-12)
    sc = {"type": "yarn", "factor": 8.0, "original_length": 4096}
    yarn, mag = T.rotary_theta(dict(a, scaling=sc))
    assert mag == pytest.approx(0.1 * math.log(8) + 1)
    turns = 4096 * plain / (2 * math.pi)
    # (the ramp is over whole pairs: it may begin and end one pair away from the bounds)
    assert np.array_equal(yarn[turns > 32 * 1.4], plain[turns > 32 * 1.4])
    assert np.allclose(yarn[turns < 1 / 1.4], plain[turns < 1 / 1.4] / 8)
    assert T.rotary_theta(dict(a, scaling=dict(sc, attention_factor=1.0)))[1] == 1.0


def test_qk_norm_unit_mean_square():
    x = _rng(5).normal(size=(3, 2, 32)) * 7
    y = T.qk_norm(x, np.ones(32), 0.0)
    assert np.allclose((y * y).mean(axis=-1), 1.0)
    assert T.qk_norm(np.zeros((1, 8)), np.ones(8), 1e-6).tolist() == [[0.0] * 8]


def test_attention_against_scalar_loops():
    r = _rng(6)
    b, lq, lk, h, kv, d = 3, 4, 5, 4, 2, 8
    q, k, v = r.normal(size=(b * lq, 8 + h * d)), r.normal(size=(b * lk, kv * d)), r.normal(size=(b * lk, 16 + kv * d))
    lens = [5, 2, 0]
    for causal in (False, True):
        attrs = {"batch": b, "heads": h, "kv_heads": kv, "head_dim": d, "causal": causal, "q_col": 8, "v_col": 16}
        y = T.attention(attrs, q, k, v, lens)
        for i in range(b):
            for t in range(lq):
                for j in range(h):
                    g = j // 2
                    keys = [n for n in range(lens[i]) if not causal or n <= lens[i] - lq + t]
                    s = [sum(q[i * lq + t, 8 + j * d + e] * k[i * lk + n, g * d + e] for e in range(d)) / math.sqrt(d)
                         for n in keys]
                    w = [math.exp(x) for x in s]
                    for e in range(d):
                        ref = sum(p * v[i * lk + n, 16 + g * d + e] for p, n in zip(w, keys)) / sum(w) if keys else 0.0
                        assert y[i * lq + t, j * d + e] == pytest.approx(ref, rel=1e-11, abs=1e-13)


def test_attention_ignores_what_is_past_the_lengths():
    r = _rng(7)
    attrs = {"batch": 2, "heads": 2, "head_dim": 8}
    q, k, v = (r.normal(size=(2 * n, 16)) for n in (3, 6, 6))
    a = T.attention(attrs, q, k, v, [4, 0])
    k2, v2 = k.copy(), v.copy()
    for t in (k2, v2):
        t[4:6], t[6:] = np.nan, np.inf
    b = T.attention(attrs, q, k2, v2, [4, 0])
    assert np.array_equal(a, b) and not a[3:].any()


def test_run_graph_reads_index_inputs():
    g = {"inputs": [{"name": "x", "shape": [2, 8], "dtype": "bf16"}, {"name": "p", "shape": [2], "dtype": "i32"}],
         "nodes": [{"name": "y", "composite": "rotary", "inputs": ["x", "p"], "out_dtype": "bf16",
                    "attrs": {"heads": 1, "head_dim": 8}}],
         "outputs": [{"name": "y"}]}
    x = np.ones((2, 8))
    # (a position that bf16 does not hold stays whole)
    y = oracle.run_graph(g, [], [x, [1001, 0]], mode="exact")[0]
    assert y[0, 0] == pytest.approx(math.cos(1001) - math.sin(1001), abs=1e-12)
    assert np.array_equal(y[1], x[1])
