"""Operators of a step that verifies drafted tokens, in float64, op by op.

TEST INFRASTRUCTURE ONLY (see the package docstring).

mxdense         rows of x and of w in blocks of 32 columns (the last may be shorter): a block's
                values become s c with s = 2^(floor(log2 max|v|) - 2), its exponent at least -127, and c
                the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, the one with the
                even place in that list where two are as near.  The products of these values summed.
                A row that holds an infinity or a NaN gives NaN.
attention_tree  query i of sequence b sees the first clamp(lengths_b, 0, k_len) keys of its cache, and of the
                drafted keys those of the tokens on its path: i, its parent, that one's parent, ...  A parent
                that is not one of the tokens before its own ends the path.
logits          with n_t the occurrences of token t in the generated part of a sequence's history (and on a
                row's path of drafted tokens), s_t whether t occurs there or in the prompt:
                x r or x / r where s_t (x > 0: the quotient), less frequency n_t, less presence where
                n_t > 0, plus the last bias entry for t, -inf where the mask's bit is 0.  The history is its
                first clamp(length, 0, T) tokens, the prompt its first prompt_length; tokens outside
                the vocabulary count for nothing.
"""

import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _f64(a):
    return np.asarray(a, dtype=np.float64)


def mx_values(a):
    """The values that the rows' codes stand for; NaN through rows that hold an infinity or a NaN."""
    a = _f64(a)
    m, k = a.shape
    out = np.zeros_like(a)
    bad = ~np.isfinite(a).all(axis=1)
    for c in range(0, k, 32):
        v = np.where(bad[:, None], 0.0, a[:, c:c + 32])
        top = np.abs(v).max(axis=1)
        e = np.frexp(top)[1] - 1 - 2  # top = f 2^x with f in [0.5, 1)
        s = np.ldexp(1.0, np.maximum(np.where(top > 0, e, 0), -127))[:, None]
        far = np.abs(np.abs(v / s)[:, :, None] - GRID)
        # (np.argmin takes the first of equals: the even places are looked at first)
        order = [0, 2, 4, 6, 1, 3, 5, 7]
        code = np.asarray(order)[far[:, :, order].argmin(axis=2)]
        out[:, c:c + 32] = np.copysign(GRID[code] * s, v)
    out[bad] = np.nan
    return out


def mxdense(x, w, magnitudes=False):
    """With magnitudes: (output, sum of |x||w| over the codes' values)."""
    vx, vw = mx_values(x), mx_values(w)
    bad = np.isnan(vx).any(axis=1)
    vx[bad] = 0.0
    y, mag = vx @ vw.T, np.abs(vx) @ np.abs(vw).T
    y[bad] = np.nan
    return (y, mag) if magnitudes else y


def path(parents, i):
    """Drafted token i and those that lead to it."""
    got = [i]
    while 0 <= parents[got[-1]] < got[-1]:
        got.append(int(parents[got[-1]]))
    return got


def attention_tree(attrs, q, k, v, dk, dv, lengths, parents, magnitudes=False):
    """With magnitudes: (output, sum of p |v|, largest sum of scale |q||k| of each row)."""
    b, h, d = int(attrs["batch"]), int(attrs["heads"]), int(attrs["head_dim"])
    kv = int(attrs.get("kv_heads", h))
    scale = float(attrs.get("scale", 1.0 / math.sqrt(d)))
    qc, kc, vc, dkc, dvc = (int(attrs.get(n, 0)) for n in ("q_col", "k_col", "v_col", "draft_k_col", "draft_v_col"))
    q, k, v, dk, dv = (_f64(a) for a in (q, k, v, dk, dv))
    t, lk = len(q) // b, len(k) // b
    out = np.zeros((len(q), h * d))
    absum, score = np.zeros_like(out), np.zeros((len(q), h))
    for i in range(b):
        n = min(max(int(lengths[i]), 0), lk)
        tree = [int(p) for p in np.asarray(parents)[i * t:(i + 1) * t]]
        for j in range(t):
            on = [i * t + a for a in path(tree, j)]
            r = i * t + j
            for head in range(h):
                at = head // (h // kv) * d
                ks = np.concatenate([k[i * lk:i * lk + n, kc + at:kc + at + d], dk[on, dkc + at:dkc + at + d]])
                vs = np.concatenate([v[i * lk:i * lk + n, vc + at:vc + at + d], dv[on, dvc + at:dvc + at + d]])
                qs = q[r, qc + head * d:qc + (head + 1) * d]
                cols = slice(head * d, (head + 1) * d)
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (ks @ qs)
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[r, cols] = p @ vs
                    if magnitudes:
                        absum[r, cols] = p @ np.abs(vs)
                        score[r, head] = scale * (np.abs(ks) @ np.abs(qs)).max()
    return (out, absum, np.repeat(score, d, axis=1)) if magnitudes else out


def rules_of(name):
    """The rules that a composite's name lists."""
    got = name.split("_")
    rest = [r for r in ("penalties", "drafts", "bias", "mask") if r in got]
    if got != ["logits"] + rest or not rest or ("drafts" in rest and "penalties" not in rest):
        raise ValueError("unknown composite %r" % name)
    return rest


def float_params(node):
    """The names of a node's inputs that are float32 whatever the graph computes in."""
    if node["composite"].split("_")[0] != "logits":
        return []
    rules, at, got = rules_of(node["composite"]), 1, []
    if "penalties" in rules:
        got.append(node["inputs"][at + 3])
        at += 4
    if "drafts" in rules:
        at += 2
    if "bias" in rules:
        got.append(node["inputs"][at + 1])
    return got


def logits(name, attrs, x, *rest, magnitudes=False):
    """With magnitudes: (output, the size of what was added up)."""
    rules, rest, b = rules_of(name), list(rest), int(attrs["batch"])
    y = _f64(x).copy()
    m, vocab = y.shape
    rows = m // b
    mag = np.abs(y)

    def take():
        return np.asarray(rest.pop(0))

    def known(tokens):
        return [int(t) for t in tokens if 0 <= int(t) < vocab]

    if "penalties" in rules:
        history, prompts, lengths, strengths = take().reshape(b, -1), take(), take(), _f64(take())
        tree = (take().reshape(b, rows), take().reshape(b, rows)) if "drafts" in rules else None
        for i in range(b):
            n = min(max(int(lengths[i]), 0), history.shape[1])
            cut = min(max(int(prompts[i]), 0), n)
            r, presence, frequency = (float(s) for s in strengths[i])
            for j in range(rows):
                made = known(history[i, cut:n])
                if tree is not None:
                    made += known(tree[0][i, path(tree[1][i], j)])
                row = i * rows + j
                for t in set(known(history[i, :cut])) | set(made):
                    y[row, t] = y[row, t] / r if y[row, t] > 0 else y[row, t] * r
                    mag[row, t] = abs(y[row, t])
                for t in set(made):
                    y[row, t] -= frequency * made.count(t) + presence
                    mag[row, t] += 2 * abs(frequency) * made.count(t) + 2 * abs(presence)
    if "bias" in rules:
        tokens, values = take().reshape(b, -1), _f64(take())
        for i in range(b):
            for t, e in {int(t): e for e, t in enumerate(tokens[i])}.items():
                if 0 <= t < vocab:
                    y[i * rows:(i + 1) * rows, t] += values[i, e]
                    mag[i * rows:(i + 1) * rows, t] += abs(values[i, e])
    if "mask" in rules:
        words = take().astype(np.int64).reshape(m, -1)
        t = np.arange(vocab)
        y[(words[:, t // 32] >> (t % 32)) & 1 == 0] = -np.inf
    return (y, mag) if magnitudes else y
