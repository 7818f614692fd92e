"""The float64 definitions of the drafted tokens' operators, pinned to hand values, scalar loops and invariants."""

import math

import numpy as np
import pytest

import oracle
from oracle import drafts as D
from oracle import transformer as T


def test_mx_values_by_hand():
    # largest 6: s = 2^(2 - 2) = 1; halves between two codes go to the one with the even place
    row = np.array([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.2500001, 5.0000001, 0.0])
    want = [6, 0, 1, 1, 2, 2, 4, 4, 0, -0.5, 6, 0]
    assert D.mx_values(row[None])[0].tolist() == want
    # 7 of a block up to 7.99 is past the last code
    assert D.mx_values([[7.99, 7.0, -7.5]])[0].tolist() == [6, 6, -6]
    # every block by itself, the last one shorter
    a = np.zeros((1, 70))
    a[0, 0], a[0, 33], a[0, 69] = 3.0, 48.0, 2.0 ** -140
    assert D.mx_values(a)[0, [0, 33, 69]].tolist() == [3.0, 48.0, 0.0]  # (2^-140 is under half of 2^-127 / 2)
    assert D.mx_values([[2.0 ** -127, -1.5 * 2.0 ** -127]])[0].tolist() == [2.0 ** -127, -1.5 * 2.0 ** -127]


def test_mx_values_against_a_scalar_search():
    r = np.random.default_rng(1)
    a = r.normal(size=(4, 45)) * np.exp(r.normal(size=(4, 45)) * 3)
    got = D.mx_values(a)
    for m in range(4):
        for c in range(0, 45, 32):
            block = a[m, c:c + 32]
            s = 2.0 ** (math.floor(math.log2(max(abs(v) for v in block))) - 2)
            for i, v in enumerate(block):
                best = min(abs(abs(v) / s - g) for g in D.GRID)
                assert abs(abs(v) / s - abs(got[m, c + i]) / s) == pytest.approx(best, abs=1e-12)
                assert got[m, c + i] == 0 or got[m, c + i] * v > 0


def test_mxdense_of_exact_values_is_the_product():
    r = np.random.default_rng(2)
    x, w = (r.choice(np.concatenate([D.GRID, -D.GRID]), size=s) for s in ((5, 96), (7, 96)))
    x[:, ::32], w[:, ::32] = 4.0, -6.0  # every block's scale is 1
    assert np.array_equal(D.mxdense(x, w), x @ w.T)
    assert np.array_equal(D.mxdense(x * 2.0 ** 60, w * 2.0 ** -80), (x @ w.T) * 2.0 ** -20)
    x[2, 50], x[4, 0] = np.inf, np.nan
    y = D.mxdense(x, w)
    assert np.isnan(y[[2, 4]]).all() and not np.isnan(y[[0, 1, 3]]).any()


def test_path():
    parents = [-1, 0, 0, 2, 7, 4, -3, 6]  # (7 is not before 4: its path ends)
    assert [D.path(parents, i) for i in range(8)] == [[0], [1, 0], [2, 0], [3, 2, 0], [4], [5, 4], [6], [7, 6]]


def _tree(r, b, t, lk, h, kv, d):
    return (r.normal(size=(b * t, h * d)), r.normal(size=(b * lk, kv * d)), r.normal(size=(b * lk, kv * d)),
            r.normal(size=(b * t, kv * d)), r.normal(size=(b * t, kv * d)))


def test_attention_tree_chain_is_causal_attention():
    r = np.random.default_rng(3)
    b, t, lk, h, kv, d = 2, 5, 7, 4, 2, 8
    q, k, v, dk, dv = _tree(r, b, t, lk, h, kv, d)
    lengths = np.array([7, 3])
    attrs = {"batch": b, "heads": h, "kv_heads": kv, "head_dim": d}
    got = D.attention_tree(attrs, q, k, v, dk, dv, lengths, np.tile(np.arange(t) - 1, b))
    joined_k, joined_v = np.zeros((b * (lk + t), kv * d)), np.zeros((b * (lk + t), kv * d))
    for i, n in enumerate(lengths):
        for to, cache, new in ((joined_k, k, dk), (joined_v, v, dv)):
            to[i * (lk + t):i * (lk + t) + n] = cache[i * lk:i * lk + n]
            to[i * (lk + t) + n:i * (lk + t) + n + t] = new[i * t:(i + 1) * t]
    ref = T.attention(dict(attrs, causal=True), q, joined_k, joined_v, lengths + t)
    assert np.abs(got - ref).max() < 1e-13


def test_attention_tree_sees_only_its_path():
    r = np.random.default_rng(4)
    q, k, v, dk, dv = _tree(r, 1, 4, 3, 1, 1, 8)
    parents = np.array([-1, 0, 0, 1])
    attrs = {"batch": 1, "heads": 1, "head_dim": 8}
    ref = D.attention_tree(attrs, q, k, v, dk, dv, [2], parents)
    dk[2], dv[2], k[2], v[2] = np.nan, np.inf, np.inf, np.nan  # on no other's path; past the length
    got = D.attention_tree(attrs, q, k, v, dk, dv, [2], parents)
    assert np.array_equal(got[[0, 1, 3]], ref[[0, 1, 3]]) and np.isnan(got[2]).all()
    alone = D.attention_tree(attrs, q, k, v, dk, dv, [0], parents)
    assert np.allclose(alone[0], dv[0])  # an empty cache: the first token sees itself


def test_logits_by_hand():
    x = np.array([[2.0, -2.0, 1.0, 0.5, 3.0]])
    got = D.logits("logits_penalties_bias_mask", {"batch": 1}, x,
                   [0, 1, 3, 3, 9, 2], [2], [5], [[2.0, 0.25, 0.5]],    # prompt 0 1, made 3 3 (9: no token), 2 not in it yet
                   [2, 3, 2, -1], [[10.0, 1.0, 20.0, 7.0]], [0b01111])
    assert got[0].tolist() == [1.0, -4.0, 21.0, 0.25 - 1.0 - 0.25 + 1.0, -np.inf]


def test_logits_of_drafted_rows():
    x = np.ones((3, 6))
    got = D.logits("logits_penalties_drafts", {"batch": 1}, x, [4], [0], [1], [[1.0, 0.0, 1.0]],
                   [2, 2, 5], [-1, 0, 0])
    assert got.tolist() == [[1, 1, 0, 1, 0, 1], [1, 1, -1, 1, 0, 1], [1, 1, 0, 1, 0, 0]]


def test_logits_rules_one_after_another():
    """The composite with every rule is that of each alone, one after the other."""
    r = np.random.default_rng(5)
    b, rows, vocab = 2, 3, 50
    x = r.normal(size=(b * rows, vocab))
    pen = [r.integers(-2, vocab + 2, b * 9), [4, 0], [9, 5], np.abs(r.normal(size=(b, 3))) + 0.5]
    bias = [r.integers(-1, vocab, b * 4), r.normal(size=(b, 4))]
    mask = [r.integers(-2 ** 31, 2 ** 31, b * rows * 2)]
    attrs = {"batch": b}
    whole = D.logits("logits_penalties_bias_mask", attrs, x, *pen, *bias, *mask)
    step = D.logits("logits_mask", attrs, D.logits("logits_bias", attrs, D.logits("logits_penalties", attrs, x, *pen), *bias), *mask)
    assert np.array_equal(whole, step)
    node = {"composite": "logits_bias_mask", "inputs": ["x", "t", "v", "m"], "attrs": attrs, "out_dtype": "bf16"}
    assert D.float_params(node) == ["v"]
    assert np.array_equal(oracle.run_node(dict(node, out_dtype="f32"), [x] + bias + mask),
                          D.logits("logits_bias_mask", attrs, x, *bias, *mask))
    for name in ("logits", "logits_drafts", "logits_mask_bias", "logits_penalties_penalties"):
        with pytest.raises(ValueError):
            D.rules_of(name)
