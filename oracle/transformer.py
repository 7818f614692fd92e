"""Transformer-layer operators in float64, op by op.

TEST INFRASTRUCTURE ONLY (see the package docstring).

qdense     symmetric 8-bit codes of each row of x and of each row of w,
           code = rint(127 v / max|v|) (ties to even; 0 for an all-zero row), their exact
           integer products summed, times max|x_m| / 127 and max|w_n| / 127.  A
           row that holds an infinity or a NaN has no codes: its outputs are NaN.
rotary     pair i of a head turned by position * theta_i and scaled by mag; pairs
           (i, i + rd / 2) ("half") or (2 i, 2 i + 1) ("interleaved") of the first rd columns.
qk_norm    x / sqrt(mean(x^2) + eps) * weight over the columns of each head.
attention  rows of heads; key j of batch b is seen by query i while j < len_b and, causal,
           while j < len_b - q_len + i + 1; softmax over the seen keys of scale q.k, times
           the values; zero for a query that sees none.  What stands past the lengths does
           not matter.
"""

import math

import numpy as np


def _f64(a):
    return np.asarray(a, dtype=np.float64)


def row_codes(a):
    """Codes of each row and the magnitude that code 127 stands for."""
    a = _f64(a)
    top = np.abs(a).max(axis=1)
    with np.errstate(invalid="ignore", divide="ignore"):
        codes = np.rint(127.0 * a / top[:, None])
    codes[top == 0] = 0.0
    return codes, top


def qdense(x, w):
    cx, tx = row_codes(x)
    cw, tw = row_codes(w)
    scale = np.outer(tx / 127.0, tw / 127.0)
    bad = ~np.isfinite(tx)
    cx[bad] = 0.0
    with np.errstate(invalid="ignore"):
        y = (cx @ cw.T) * scale
    y[bad] = np.nan
    return y


def rotary_theta(attrs):
    """Angle per position of each pair, and the factor on the rotated values."""
    rd = int(attrs.get("rotary_dim", attrs["head_dim"]))
    base = float(attrs.get("base", 10000.0))
    sc = attrs.get("scaling")
    kind = sc["type"] if sc else None
    factor = float(sc["factor"]) if sc else 1.0
    if kind == "ntk" and rd > 2:
        base *= factor ** (rd / (rd - 2.0))
    i = np.arange(rd // 2, dtype=np.float64)
    theta = base ** (-2.0 * i / rd)
    if kind == "linear":
        return theta / factor, 1.0
    if kind != "yarn":
        return theta, 1.0
    length = float(sc["original_length"])

    def pair_of(turns):
        # the pair that turns `turns` times over the original length
        return rd * math.log(length / (turns * 2.0 * math.pi)) / (2.0 * math.log(base))

    low = max(math.floor(pair_of(float(sc.get("beta_fast", 32.0)))), 0)
    high = min(math.ceil(pair_of(float(sc.get("beta_slow", 1.0)))), rd - 1)
    slow = np.clip((i - low) / max(high - low, 1e-3), 0.0, 1.0)
    return theta * (1.0 - slow) + theta / factor * slow, float(sc.get("attention_factor", 0.1 * math.log(factor) + 1.0))


def qk_norm(x, weight, eps):
    """x [..., D]."""
    x = _f64(x)
    return x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * _f64(weight)


def rotate(x, positions, theta, mag, interleaved):
    """x [M, heads, D]; the first 2 len(theta) columns turn."""
    x = _f64(x)
    n = len(theta)
    angle = _f64(positions)[:, None] * theta
    c, s = (np.cos(angle) * mag)[:, None], (np.sin(angle) * mag)[:, None]
    y = x.copy()
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def rotary(attrs, x, positions, weights=None):
    h, kv, d = int(attrs["heads"]), int(attrs.get("kv_heads", 0)), int(attrs["head_dim"])
    theta, mag = rotary_theta(attrs)
    x = _f64(x)[:, :(h + kv) * d].reshape(len(x), h + kv, d).copy()
    if weights is not None:
        eps = float(attrs.get("eps", 1e-6))
        x[:, :h] = qk_norm(x[:, :h], weights[0], eps)
        if kv:
            x[:, h:] = qk_norm(x[:, h:], weights[1], eps)
    return rotate(x, positions, theta, mag, attrs.get("layout", "half") == "interleaved").reshape(len(x), -1)


def attention(attrs, q, k, v, lengths=None, magnitudes=False):
    """With magnitudes: (output, sum of p |v|, largest sum of scale |q||k| of each row),
    what the rounding bounds of a computed result are made of."""
    b, h, d = int(attrs["batch"]), int(attrs["heads"]), int(attrs["head_dim"])
    kv = int(attrs.get("kv_heads", h))
    scale = float(attrs.get("scale", 1.0 / math.sqrt(d)))
    qc, kc, vc = (int(attrs.get(n, 0)) for n in ("q_col", "k_col", "v_col"))
    q, k, v = _f64(q), _f64(k), _f64(v)
    lq, lk = len(q) // b, len(k) // b
    out = np.zeros((len(q), h * d))
    absum, score = np.zeros_like(out), np.zeros((len(q), h))
    for i in range(b):
        n = lk if lengths is None else min(max(int(lengths[i]), 0), lk)
        for t in range(lq):
            seen = n if not attrs.get("causal", False) else min(n, n - lq + t + 1)
            if seen <= 0:
                continue
            r = i * lq + t
            for j in range(h):
                g = j // (h // kv)
                ks = k[i * lk:i * lk + seen, kc + g * d:kc + (g + 1) * d]
                vs = v[i * lk:i * lk + seen, vc + g * d:vc + (g + 1) * d]
                qs = q[r, qc + j * d:qc + (j + 1) * d]
                s = scale * (ks @ qs)
                with np.errstate(invalid="ignore", over="ignore"):
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[r, j * d:(j + 1) * d] = p @ vs
                    if magnitudes:
                        absum[r, j * d:(j + 1) * d] = p @ np.abs(vs)
                        score[r, j] = scale * (np.abs(ks) @ np.abs(qs)).max()
    return (out, absum, np.repeat(score, d, axis=1)) if magnitudes else out
