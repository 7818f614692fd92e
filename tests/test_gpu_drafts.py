"""Parity of the drafted tokens' composites with their float64 definitions, at the sizes, types, lengths, trees and
masks where they can go wrong.

Rounding bounds (u = 2^-8 for bf16, e = 2^-24 for float32):
mxdense         codes and scales are exact; K terms are summed in float32, each addition off by 2 e of the sum of
                magnitudes at most (the matrix instructions may cut off instead of rounding); bias, residual and
                activation cost a few e of the terms, GELU 2^-18 of them; the bf16 output u of the result.
attention_tree  as attention: a score is off by (D + 8) e sum |q||k| scale, which moves its weight by as
                much relatively, in numerator and denominator; the sums over n keys add (n + 200) e; in bf16
                each weight is rounded (u of sum p |v|) and the result again.
logits          six operations of float32, each off by e of what it gives; the bf16 output u of the result.
"""

import numpy as np
import pytest

import oracle
from oracle import drafts as D
from paper_2105_03215_amd import workloads
from paper_2105_03215_amd.workloads import to_bf16_values
from parity_util import announce
from test_gpu_transformer import DEV, E, U, _close, _normal

pytestmark = pytest.mark.gpu


def _engine(composite, ins, args, attrs, dtype, consts=()):
    """ins: name -> (host array, dtype)."""
    from paper_2105_03215_amd import capi
    g = {"format": "byoc-subgraph", "version": 1,
         "inputs": [{"name": n, "shape": list(a.shape), "dtype": d} for n, (a, d) in ins.items()],
         "constants": [{"name": n, "index": i, "shape": list(a.shape), "dtype": "f32"} for i, (n, a) in enumerate(consts)],
         "nodes": [{"name": "y", "composite": composite, "inputs": list(args), "attrs": attrs, "out_dtype": dtype}],
         "outputs": [{"name": "y", "dtype": dtype}]}
    return capi.Subgraph(g, [a for _, a in consts], device=0)


def _run(composite, ins, args, attrs, dtype, consts=()):
    from paper_2105_03215_amd import runtime
    with _engine(composite, ins, args, attrs, dtype, consts) as sg:
        arrays = [a for a, _ in ins.values()]
        out = runtime.run_once(sg, arrays, DEV)[0]
        again = runtime.run_once(sg, arrays, DEV)[0]
    assert np.array_equal(out, again, equal_nan=True)  # run to run identical
    return out


# ---- mxdense -------------------------------------------------------------------

MXDENSE = [
    # m, k, n, dtype, suffix
    (1, 1, 1, "bf16", "_bias"),
    (1, 1, 1, "f32", ""),
    (1, 31, 8, "bf16", ""),
    (1, 1024, 4096, "bf16", "_bias_gelu"),
    (2, 33, 24, "f32", "_bias_add_relu"),
    (3, 129, 257, "bf16", "_bias"),
    (5, 300, 1003, "f32", "_bias_add"),
    (8, 1000, 4096, "bf16", "_bias"),
    (13, 768, 300, "bf16", "_add_leaky"),
    (16, 512, 128, "f32", "_relu6"),
    (16, 513, 96, "bf16", "_bias"),
    (17, 520, 72, "bf16", "_bias"),
    (9, 4097, 64, "bf16", "_bias"),
    (32, 2304, 4096, "bf16", "_add"),
    (32, 384, 4104, "bf16", "_add"),
    (33, 2000, 64, "f32", "_gelu"),
    (63, 2048, 40, "bf16", "_bias"),
    (65, 384, 136, "bf16", ""),
    (130, 257, 131, "f32", "_bias"),
    (200, 8200, 64, "bf16", "_bias"),
    (301, 515, 1003, "f32", "_bias_add"),
    (300, 128, 520, "bf16", "_bias_add_gelu"),
    (513, 130, 2305, "bf16", "_add"),
    (2100, 256, 8000, "bf16", "_add"),
    (2100, 130, 2300, "f32", "_bias_add"),
]


def _mx_case(m, k, n, dtype, suffix, seed=0):
    r = np.random.default_rng(m * 1000003 + k * 101 + n + seed)
    # magnitudes over a few octaves, so that blocks' scales differ
    x = to_bf16_values(_normal(r, m, k) * np.exp2(r.integers(-6, 7, (m, k))).astype(np.float32))
    w = to_bf16_values(_normal(r, n, k, std=0.05) * np.exp2(r.integers(-3, 4, (n, 1))).astype(np.float32))
    if dtype == "f32":
        x = (x * (1 + r.random((m, k)) * 2.0 ** -9)).astype(np.float32)
    if m > 2:
        x[1] = 0
    if n > 2:
        w[2] = 0
    if k > 40:
        x[0, 32:64] = 0
    return r, x, w


@pytest.mark.parametrize("m, k, n, dtype, suffix", MXDENSE)
def test_mxdense(m, k, n, dtype, suffix):
    announce("mxdense%s %dx%dx%d %s" % (suffix, m, k, n, dtype))
    r, x, w = _mx_case(m, k, n, dtype, suffix)
    ins, args, consts, rest = {"x": (x, dtype)}, ["x", "w"], [("w", w)], []
    b, res = r.normal(size=n).astype(np.float32), _normal(r, m, n)
    y, mag = D.mxdense(x, w, magnitudes=True)
    if "_bias" in suffix:
        consts.append(("b", b))
        args.append("b")
        rest.append(b)
        mag = mag + np.abs(b)
    if "_add" in suffix:
        ins["r"] = (res, dtype)
        args.append("r")
        rest.append(res)
        mag = mag + np.abs(res)
    attrs = {"alpha": 0.2} if "leaky" in suffix else {}
    got = _run("mxdense" + suffix, ins, args, attrs, dtype, consts)
    ref = oracle.run_node({"composite": "mxdense" + suffix, "attrs": attrs, "out_dtype": dtype}, [x, w] + rest, mode="exact")
    _close(got, ref, ((k + 8) * 2 * E + (2.0 ** -18 if "gelu" in suffix else 0)) * mag + 1e-37, dtype)


@pytest.mark.parametrize("tile", range(7))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_mxdense_every_tile(tile, dtype, monkeypatch):
    """Each product tile, at sizes that leave its last tiles and stages part empty."""
    monkeypatch.setenv("BYOC_MXDENSE_TILE", str(tile))
    test_mxdense(270, 1300, 330, dtype, "_bias_add")
    test_mxdense(33, 40, 40, dtype, "_bias")


@pytest.mark.parametrize("tile, m, k, n, suffix", [
    (0, 4400, 520, 4400, "_bias_add"), (0, 4400, 520, 4400, "_gelu"), (1, 2600, 1100, 4400, "_bias"),
    (2, 2100, 1100, 2100, "_bias_add_relu"), (3, 3000, 1100, 3000, ""), (4, 3000, 1100, 1700, "_add"),
    (5, 1500, 1100, 1500, "_bias_add_leaky"), (6, 800, 2100, 800, "_bias"),
])
def test_mxdense_more_tiles_than_workgroups(tile, m, k, n, suffix, monkeypatch):
    """Workgroups that take several tiles, whose ring goes on from one to the next."""
    monkeypatch.setenv("BYOC_MXDENSE_TILE", str(tile))
    test_mxdense(m, k, n, "bf16", suffix)


def test_mxdense_exact_products_are_exact():
    """Values on the grid: sums of few bits, which float32 holds whatever the order of the additions."""
    r = np.random.default_rng(5)
    grid = np.concatenate([D.GRID, -D.GRID])
    for m, k, n in ((7, 512, 96), (100, 1024, 160)):
        x, w = r.choice(grid, size=(m, k)).astype(np.float32), r.choice(grid, size=(n, k)).astype(np.float32)
        x[:, ::32], w[:, ::32] = 6, 4
        assert np.array_equal(_run("mxdense", {"x": (x, "f32")}, ["x", "w"], {}, "f32", [("w", w)]),
                              x.astype(np.float64) @ w.astype(np.float64).T)


def test_mxdense_codes_of_every_fraction():
    """One value of a block at a time against a weight of one: its code, at and next to every middle
    between two codes, in both types (bf16 where it has the value)."""
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0]
    v = [s * f for f in mids for s in (1, -1)]
    v += [float(np.nextafter(np.float32(f), np.float32(t))) for f in mids for t in (0, 9)] + [0.1, 0.26, 2.9, 6.5, 7.75]
    v = np.array(v, np.float32)
    x = np.zeros((len(v), 64), np.float32)
    x[:, 0], x[:, 40] = 4.0, 2.0 ** -100  # block scales 1 and 2^-102
    x[:, 9] = v
    w = np.zeros((8, 64), np.float32)
    w[0, 9], w[1, 0], w[2, 40] = 1, 1, 2.0 ** 100
    for dtype in ("f32", "bf16"):
        a = x if dtype == "f32" else to_bf16_values(x)
        ref = D.mxdense(a, w)
        assert np.array_equal(_run("mxdense", {"x": (a, dtype)}, ["x", "w"], {}, dtype, [("w", w)]), ref)


@pytest.mark.parametrize("m", [1, 9, 70])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_mxdense_odd_rows(m, dtype):
    """Rows of zeros, of one value, with infinities and NaN, of the smallest and largest magnitudes."""
    r = np.random.default_rng(12)
    k, n = 200, 72
    w = _normal(r, n, k)
    rows = [np.zeros(k), np.full(k, -3.0), r.normal(size=k) * 1e-39, r.normal(size=k) * 2.0 ** -126,
            r.normal(size=k) * 2.0 ** 120, np.where(np.arange(k) == 77, np.inf, 1.0),
            np.where(np.arange(k) == 199, np.nan, 1.0), np.where(np.arange(k) == 0, -np.inf, 0.0),
            np.full(k, 1.99 * 2.0 ** 127)]
    for i, row in enumerate(rows):
        x = _normal(r, m, k)
        with np.errstate(over="ignore"):
            x[(3 * i) % m] = to_bf16_values(row.astype(np.float32))
            y = _run("mxdense", {"x": (x, dtype)}, ["x", "w"], {}, dtype, [("w", w)])
            ref, mag = D.mxdense(x, w, magnitudes=True)
        # (where the terms' magnitudes sum to more than float32 holds, partial sums of either sign may overflow, and an
        # infinity less an infinity is a NaN: nothing is said of those; and sums of float32 denormals may flush: an
        # absolute slack of the smallest normal)
        held = ~(mag > 3e38)
        assert held.mean() > 0.1 or m == 1
        _close(np.where(held, y, 0), np.where(held, ref, 0), np.where(held, (k + 8) * 2 * E * mag, 0) + 2.0 ** -126, dtype)


def test_mxdense_weights_of_no_finite_value():
    """A channel whose weights hold an infinity or a NaN is NaN, its neighbours are not."""
    r = np.random.default_rng(13)
    w = _normal(r, 40, 96)
    w[7, 50], w[20, 0] = np.inf, np.nan
    for m in (3, 50):
        y = _run("mxdense", {"x": (_normal(r, m, 96), "bf16")}, ["x", "w"], {}, "bf16", [("w", w)])
        assert np.isnan(y[:, [7, 20]]).all() and np.isfinite(np.delete(y, [7, 20], axis=1)).all()


def test_mxdense_odd_widths_between_layers():
    """Rows of a width that is no multiple of 8, as input, residual, between layers and twice an output; two products
    of one value share its codes."""
    from paper_2105_03215_amd import capi, runtime
    g = workloads.GraphBuilder("t", 97)
    x = g.input("x", [41, 77], "normal")
    r = g.input("r", [41, 131], "normal")
    h = g.mxdense(x, 131, act="relu", residual=r)
    y, z = g.mxdense(h, 53, act="gelu"), g.mxdense(h, 200)
    for v in (y, h, y, z):
        g.output(v)
    wl = g.finish()
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        assert [l["name"] for l in sg.launches()].count("mx_rows") == 2  # (x's and h's)
        assert {l["kind"] for l in sg.launches()} <= {"mxdense", "transform"}
        got = runtime.run_once(sg, wl.inputs, DEV)
    vals = {"x": wl.inputs[0], "r": wl.inputs[1]}
    by = {c["name"]: wl.consts[c["index"]] for c in wl.graph["constants"]}
    for node, v in zip(wl.graph["nodes"], (got[1], got[0], got[3])):
        args = [vals.get(a, by.get(a)) for a in node["inputs"]]
        mag = D.mxdense(args[0], args[1], magnitudes=True)[1] + 20
        _close(v, oracle.run_node(node, args, mode="exact"), 2.0 ** -14 * mag, "bf16")
        vals[node["name"]] = v
    assert np.array_equal(got[0], got[2])


# ---- attention of a tree ----------------------------------------------------------

TREE = [
    # batch, drafts, k_len, heads, kv, d, dtype, lengths, tree
    (1, 1, 1, 1, 1, 8, "bf16", [0], "random"),
    (1, 1, 1, 1, 1, 8, "f32", [1], "random"),
    (2, 1, 33, 4, 1, 64, "bf16", [33, 0], "random"),
    (2, 8, 31, 2, 2, 64, "bf16", [31, 7], "random"),
    (1, 8, 300, 12, 12, 64, "bf16", [300], "random"),
    (3, 5, 700, 8, 2, 128, "bf16", [700, 1, 129], "random"),
    (3, 5, 700, 8, 2, 128, "f32", [700, 1, 129], "random"),
    (2, 32, 5000, 2, 2, 80, "bf16", [5000, 4097], "random"),
    (2, 32, 64, 3, 3, 64, "f32", [64, 32], "chain"),
    (2, 33, 64, 3, 3, 64, "bf16", [64, 63], "chain"),
    (1, 40, 90, 2, 2, 256, "f32", [77], "random"),
    (1, 20, 90, 2, 1, 256, "bf16", [90], "random"),
    (1, 70, 90, 2, 1, 256, "bf16", [90], "star"),
    (2, 64, 64, 4, 2, 64, "bf16", [64, 1], "random"),
    (2, 65, 257, 3, 3, 96, "bf16", [200, 257], "random"),
    (2, 61, 129, 20, 4, 160, "bf16", [100, 0], "random"),
    (1, 256, 130, 2, 1, 128, "bf16", [130], "chain"),
    (1, 256, 5, 1, 1, 32, "bf16", [5], "random"),
    (1, 255, 40, 1, 1, 64, "f32", [33], "chain"),
    (41, 33, 70, 8, 8, 64, "bf16", None, "random"),       # tiles of 128 rows, 64 columns
    (16, 40, 60, 8, 8, 48, "f32", None, "random"),        # fp32 tiles
    (70, 3, 90, 2, 1, 64, "bf16", None, "random"),        # more sequences than lanes
    (70, 20, 1500, 4, 1, 64, "bf16", None, "random"),     # the same, on the tiles
    (3, 24, 3000, 8, 2, 128, "bf16", [0, 2999, 64], "random"),  # split key axes, one of them of drafted keys alone
    (2, 2, 100, 1, 1, 32, "bf16", [101, 2 ** 31 - 1], "random"),  # lengths outside [0, k_len] are taken as its ends
    (2, 3, 100, 1, 1, 24, "bf16", [-5, 100], "random"),
]


def _parents(r, batch, t, kind):
    if kind == "chain":
        one = np.arange(t) - 1
        return np.tile(one, batch).astype(np.int32)
    if kind == "star":
        return np.tile(np.where(np.arange(t) == 0, -1, 0), batch).astype(np.int32)
    return np.concatenate([[r.integers(-1, i) if i else -1 for i in range(t)] for _ in range(batch)]).astype(np.int32)


def _tree_case(batch, t, lk, h, kv, d, lengths, kind, seed=0, packed=False):
    r = np.random.default_rng(batch * 31 + t * 1009 + lk * 7 + d + seed)
    if lengths is None:
        lengths = r.integers(0, lk + 1, batch)
    a = {"q": _normal(r, batch * t, h * d), "k": _normal(r, batch * lk, kv * d), "v": _normal(r, batch * lk, kv * d),
         "dk": _normal(r, batch * t, kv * d), "dv": _normal(r, batch * t, kv * d)}
    a["n"], a["p"] = np.array(lengths, dtype=np.int64).astype(np.int32), _parents(r, batch, t, kind)
    return a, {"batch": batch, "heads": h, "kv_heads": kv, "head_dim": d}


def _check_tree(a, attrs, dtype, y=None):
    ins = {n: (v, "i32" if v.dtype == np.int32 else dtype) for n, v in a.items()}
    if y is None:
        y = _run("attention_tree", ins, list(ins), attrs, dtype)
    ref, absum, score = D.attention_tree(attrs, *a.values(), magnitudes=True)
    d, n = attrs["head_dim"], len(a["k"]) // attrs["batch"] + len(a["q"]) // attrs["batch"]
    bound = (2 * (d + 8) * E * score + (n + 200) * E + (U if dtype == "bf16" else 0)) * absum
    _close(y, ref, bound, dtype)
    return y


@pytest.mark.parametrize("batch, t, lk, h, kv, d, dtype, lengths, kind", TREE)
def test_attention_tree(batch, t, lk, h, kv, d, dtype, lengths, kind):
    announce("attention_tree b %d t %d k %d heads %d/%d d %d %s %s" % (batch, t, lk, h, kv, d, dtype, kind))
    a, attrs = _tree_case(batch, t, lk, h, kv, d, lengths, kind)
    _check_tree(a, attrs, dtype)


@pytest.mark.parametrize("batch, t, lk, h, kv, d, dtype", [
    (2, 9, 200, 4, 2, 64, "bf16"), (2, 9, 200, 4, 2, 64, "f32"), (2, 40, 100, 4, 2, 64, "bf16"),
    (2, 40, 100, 4, 2, 128, "bf16"), (2, 70, 300, 2, 1, 72, "bf16"), (16, 40, 60, 8, 8, 64, "f32"),
    (2, 30, 3000, 4, 1, 128, "bf16"),
])
def test_attention_tree_hidden_places_do_not_matter(batch, t, lk, h, kv, d, dtype):
    """Infinities and NaN in the cache past a sequence's length, and in drafted keys and values: the rows that do not
    see them are as the definition has them, the others NaN or infinite as it says."""
    a, attrs = _tree_case(batch, t, lk, h, kv, d, [lk - 3] + [17 % lk] * (batch - 1), "random", seed=3)
    for i in range(batch):
        n = int(a["n"][i])
        a["k"][i * lk + n:(i + 1) * lk] = np.nan
        a["v"][i * lk + n:(i + 1) * lk] = np.inf
    # the last token of each sequence is on no other's path, nor is one without children
    for i in range(batch):
        p = a["p"][i * t:(i + 1) * t]
        leaves = sorted(set(range(t)) - set(p.tolist()))
        a["dv"][i * t + leaves[-1]] = np.nan
        a["dk"][i * t + leaves[0]] = np.nan
        a["dv"][i * t + leaves[len(leaves) // 2], ::3] = np.inf
    with np.errstate(invalid="ignore"):
        y = _check_finite_rows(a, attrs, dtype)
    assert np.isnan(y[leaves[-1] - t]).all()


def _check_finite_rows(a, attrs, dtype):
    ins = {n: (v, "i32" if v.dtype == np.int32 else dtype) for n, v in a.items()}
    y = _run("attention_tree", ins, list(ins), attrs, dtype)
    ref, absum, score = D.attention_tree(attrs, *a.values(), magnitudes=True)
    d, n = attrs["head_dim"], len(a["k"]) // attrs["batch"]
    ok = np.isfinite(ref)
    assert np.isfinite(y[ok]).all() and not np.isfinite(y[~ok]).any()
    bound = (2 * (d + 8) * E * score + (n + 500) * E + (U if dtype == "bf16" else 0)) * absum
    _close(np.where(ok, y, 0), np.where(ok, ref, 0), np.where(ok, bound, 0), dtype)
    return y


@pytest.mark.parametrize("t, d, dtype", [(7, 64, "bf16"), (100, 64, "bf16"), (100, 32, "f32")])
def test_attention_tree_parents_of_any_value(t, d, dtype):
    """A parent that is not before its token - the token itself, a later one, one of no sequence - ends the path."""
    a, attrs = _tree_case(2, t, 50, 2, 1, d, [50, 20], "random", seed=9)
    p = a["p"]
    p[0], p[3], p[5], p[t], p[t + 2], p[t + 4] = 5, 3, 6, 2 ** 31 - 1, -2 ** 31, t
    _check_tree(a, attrs, dtype)


def test_attention_tree_packed_rows():
    """Queries, keys and values side by side in rows, the drafted ones too, with columns that are not theirs; rows of
    the cache and of the drafted tokens are different distances apart."""
    r = np.random.default_rng(21)
    for dtype, t, d in (("bf16", 40, 64), ("bf16", 6, 128), ("f32", 6, 40), ("bf16", 50, 136)):
        h, kv, lk, b = 6, 2, 150, 2
        qkv, cache = _normal(r, b * t, (h + 2 * kv) * d + 16), _normal(r, b * lk, 2 * kv * d + 8)
        attrs = {"batch": b, "heads": h, "kv_heads": kv, "head_dim": d, "q_col": 8, "k_col": kv * d + 8, "v_col": 0,
                 "draft_k_col": 8 + h * d, "draft_v_col": 8 + (h + kv) * d, "scale": 0.07}
        n, p = np.array([150, 33], np.int32), _parents(r, b, t, "random")
        ins = {"x": (qkv, dtype), "c": (cache, dtype), "n": (n, "i32"), "p": (p, "i32")}
        y = _run("attention_tree", ins, ["x", "c", "c", "x", "x", "n", "p"], attrs, dtype)
        _check_tree({"q": qkv, "k": cache, "v": cache, "dk": qkv, "dv": qkv, "n": n, "p": p}, attrs, dtype, y)


def test_attention_tree_chain_is_causal_attention():
    """A chain of drafted tokens over a cache against causal self attention over both together."""
    b, t, lk, h, kv, d = 2, 21, 90, 4, 2, 64
    a, attrs = _tree_case(b, t, lk, h, kv, d, [90, 44], "chain", seed=4)
    y = _check_tree(a, attrs, "f32")
    k, v = np.zeros((b * (lk + t), kv * d), np.float32), np.zeros((b * (lk + t), kv * d), np.float32)
    for i, n in enumerate(a["n"]):
        for to, cache, new in ((k, "k", "dk"), (v, "v", "dv")):
            to[i * (lk + t):i * (lk + t) + n] = a[cache][i * lk:i * lk + n]
            to[i * (lk + t) + n:i * (lk + t) + n + t] = a[new][i * t:(i + 1) * t]
    ins = {"q": (a["q"], "f32"), "k": (k, "f32"), "v": (v, "f32"), "n": ((a["n"] + t).astype(np.int32), "i32")}
    z = _run("attention_lengths", ins, list(ins), dict(attrs, causal=True), "f32")
    assert np.abs(y - z).max() <= 2.0 ** -17


# ---- rules on logits ----------------------------------------------------------------

RULES = [
    # batch, rows, vocab, history, entries, dtype, rules
    (1, 1, 1, 1, 1, "f32", "penalties_bias_mask"),
    (1, 1, 7, 3, 2, "bf16", "penalties"),
    (1, 1, 32000, 200, 0, "f32", "penalties"),
    (2, 3, 33, 5, 3, "f32", "penalties_bias_mask"),
    (3, 1, 4096, 300, 0, "bf16", "mask"),
    (3, 1, 4097, 300, 20, "bf16", "bias"),
    (2, 2, 5003, 1000, 40, "bf16", "bias_mask"),
    (5, 1, 8200, 2000, 0, "bf16", "penalties_mask"),
    (2, 1, 1003, 5000, 300, "f32", "penalties_bias"),
    (1, 1, 300, 9, 0, "f32", "penalties_drafts"),
    (3, 7, 2050, 60, 9, "bf16", "penalties_drafts_bias_mask"),
    (2, 64, 515, 40, 0, "f32", "penalties_drafts_mask"),
    (1, 256, 70, 20, 5, "bf16", "penalties_drafts_bias"),
    (2, 257, 65, 20, 0, "f32", "penalties"),
    (4, 2, 50257, 700, 12, "f32", "penalties_drafts_bias_mask"),
    (130, 1, 260, 33, 2, "bf16", "penalties_bias_mask"),
    (2, 1, 20000, 9000, 2500, "bf16", "penalties_bias_mask"),    # lists that no registers and no LDS hold
    (120, 1, 150000, 40, 6, "bf16", "penalties_bias_mask"),      # chunks that follow one another in a workgroup
    (24, 16, 50257, 30, 3, "f32", "penalties_drafts_bias"),      # the same of rows
    (300, 1, 70001, 1, 0, "bf16", "mask"),
]


def _rules_case(batch, rows, vocab, history, entries, dtype, rules, seed=0):
    r = np.random.default_rng(vocab * 13 + batch + rows + seed)
    m = batch * rows
    x = (r.normal(size=(m, vocab)) * 4).astype(np.float32)
    ins = {"x": (to_bf16_values(x) if dtype == "bf16" else x, dtype)}

    def tokens(n):  # often the same, some of no token
        t = (r.random(n) ** 3 * vocab).astype(np.int64)
        return np.where(r.random(n) < 0.05, r.choice([-1, vocab, 2 ** 31 - 1, -2 ** 31], n), t).astype(np.int32)

    if "penalties" in rules:
        lengths = r.integers(0, history + 1, batch)
        lengths[0] = history
        ins["h"] = (tokens(batch * history), "i32")
        ins["pl"] = (r.integers(0, lengths + 1).astype(np.int32), "i32")
        ins["n"] = (lengths.astype(np.int32), "i32")
        s = np.stack([1 + r.random(batch), 2 * r.random(batch) - 1, r.random(batch)], axis=1)
        ins["s"] = (s.astype(np.float32), "f32")
    if "drafts" in rules:
        ins["t"] = (tokens(m), "i32")
        ins["p"] = (_parents(r, batch, rows, "random"), "i32")
    if "bias" in rules:
        ins["bt"] = (tokens(batch * entries), "i32")
        ins["bv"] = ((r.normal(size=(batch, entries)) * 10).astype(np.float32), "f32")
    if "mask" in rules:
        w = r.integers(-2 ** 31, 2 ** 31, (m, (vocab + 31) // 32))
        w[0::3] = -1
        w[m - 1] = 0 if m > 1 else w[m - 1]  # a row that may take no token
        ins["m"] = (w.astype(np.int32).reshape(-1), "i32")
    return ins


def _check_rules(ins, batch, rules, dtype):
    got = _run("logits_" + rules, ins, list(ins), {"batch": batch}, dtype)
    ref, mag = D.logits("logits_" + rules, {"batch": batch}, *[a for a, _ in ins.values()], magnitudes=True)
    assert np.array_equal(got == -np.inf, ref == -np.inf)
    hidden = ref == -np.inf
    _close(np.where(hidden, 0, got), np.where(hidden, 0, ref), 6 * E * mag, dtype)
    return got


@pytest.mark.parametrize("batch, rows, vocab, history, entries, dtype, rules", RULES)
def test_logits(batch, rows, vocab, history, entries, dtype, rules):
    announce("logits_%s b %d rows %d vocab %d history %d %s" % (rules, batch, rows, vocab, history, dtype))
    _check_rules(_rules_case(batch, rows, vocab, history, entries, dtype, rules), batch, rules, dtype)


def test_logits_lengths_of_any_value():
    """Lengths and prompts outside [0, history] are taken as its ends."""
    ins = _rules_case(6, 1, 90, 25, 0, "f32", "penalties")
    for n, cut in ((np.array([-3, 0, 26, 2 ** 31 - 1, 25, 5]), np.array([5, 1, -7, 2 ** 31 - 1, -2 ** 31, 9])),):
        ins["n"], ins["pl"] = (n.astype(np.int32), "i32"), (cut.astype(np.int32), "i32")
        _check_rules(ins, 6, "penalties", "f32")


def test_logits_one_token_for_all():
    """Every place of a long history and every bias entry names one token: it counts each, and the last entry."""
    ins = _rules_case(2, 3, 200, 70000, 500, "f32", "penalties_drafts_bias", seed=1)
    for name in ("h", "t", "bt"):
        ins[name] = (np.full_like(ins[name][0], 131), "i32")
    ins["n"] = (np.array([70000, 69999], np.int32), "i32")
    ins["pl"] = (np.array([0, 3], np.int32), "i32")
    _check_rules(ins, 2, "penalties_drafts_bias", "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_every_token_met(dtype):
    """More tokens of a chunk met than are listed."""
    ins = _rules_case(2, 3, 9000, 12000, 40, dtype, "penalties_drafts_bias_mask")
    r = np.random.default_rng(3)
    ins["h"] = (np.concatenate([r.permutation(12000) % 9000 for _ in range(2)]).astype(np.int32), "i32")
    ins["n"], ins["pl"] = (np.array([12000, 11000], np.int32), "i32"), (np.array([4000, 0], np.int32), "i32")
    _check_rules(ins, 2, "penalties_drafts_bias_mask", dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_of_no_finite_value(dtype):
    """Infinities and NaN among the logits: under the mask they are -inf, elsewhere what the arithmetic gives."""
    ins = _rules_case(2, 2, 300, 40, 8, dtype, "penalties_bias_mask")
    x = ins["x"][0]
    x[:, 5::17], x[:, 6::17], x[:, 7::17] = np.nan, np.inf, -np.inf
    with np.errstate(invalid="ignore"):
        got = _run("logits_penalties_bias_mask", ins, list(ins), {"batch": 2}, dtype)
        ref, mag = D.logits("logits_penalties_bias_mask", {"batch": 2}, *[a for a, _ in ins.values()], magnitudes=True)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    flat = ~np.isfinite(ref)
    assert np.array_equal(got[flat], ref[flat], equal_nan=True)
    _close(np.where(flat, 0, got), np.where(flat, 0, ref), np.where(flat, 0, 6 * E * mag), dtype)


def test_logits_strengths_stay_float32():
    """In a bf16 graph the strengths and biases are not rounded to bf16."""
    x = np.full((1, 8), 64.0, np.float32)
    ins = {"x": (x, "bf16"), "h": (np.array([3], np.int32), "i32"), "pl": (np.array([0], np.int32), "i32"),
           "n": (np.array([1], np.int32), "i32"), "s": (np.array([[1.0, 63.998, 0.0]], np.float32), "f32"),
           "bt": (np.array([5], np.int32), "i32"), "bv": (np.array([[-63.998]], np.float32), "f32")}
    got = _run("logits_penalties_bias", ins, list(ins), {"batch": 1}, "bf16")
    want = to_bf16_values(np.float32(64) - np.float32([63.998]))[0]
    assert got[0, 3] == want and got[0, 5] == want and (np.delete(got[0], [3, 5]) == 64).all()


def test_logits_padding_columns_are_zero():
    """Rows of a width that is no multiple of 8 between a product and a dense layer, which reads the padding."""
    from paper_2105_03215_amd import capi, runtime
    import torch
    g = workloads.GraphBuilder("t", 98)
    x = g.input("x", [9, 40], "normal")
    bias = (g.index_input("bt", np.arange(9)), g.param_input("bv", np.ones((9, 1))))
    y = g.logits(g.mxdense(x, 45), 9, bias=bias)
    g.output(g.dense(y, 16))
    wl = g.finish()
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        ins, outs = runtime.inputs_for(sg, wl.inputs, DEV), runtime.outputs_for(sg, DEV)
        sg.run([torch.full_like(t, float("nan")) if t.is_floating_point() else t for t in ins], outs)  # the arena's bytes NaN
        sg.run(ins, outs)
        torch.cuda.synchronize()
        got = runtime.to_host_f64(outs[0])
    ref, vals = oracle.run_graph(wl.graph, wl.consts, wl.inputs, keep=True)
    assert np.isfinite(got).all() and np.abs(got - ref[0]).max() <= 0.05 * np.abs(ref[0]).max()


# ---- the step -------------------------------------------------------------------------

def _step(**kw):
    kw = dict(dict(batch=3, drafts=7, cached=130, hidden=256, heads=4, kv_heads=2, ffn=320, vocab=1003, history=40), **kw)
    return workloads.build("verify_step", **kw)


@pytest.mark.parametrize("kw", [dict(), dict(dtype="f32"), dict(drafts=1, batch=1), dict(batch=2, drafts=70, cached=700)])
def test_verify_step_teacher_forced(kw):
    """The composites of a step run together, each as an output of the engine, against the oracle on the
    engine's own inputs of that node."""
    from paper_2105_03215_amd import capi, runtime
    wl = _step(**kw)
    dtype = kw.get("dtype", "bf16")
    g = dict(wl.graph, outputs=[{"name": n["name"], "dtype": dtype} for n in wl.graph["nodes"]])
    with capi.Subgraph(g, wl.consts, device=0) as sg:
        outs = runtime.run_once(sg, wl.inputs, DEV)
    vals = {d["name"]: np.asarray(a, np.float64) for d, a in zip(g["inputs"], wl.inputs)}
    for c in g["constants"]:
        vals[c["name"]] = np.asarray(wl.consts[c["index"]], np.float64)
    for node, y in zip(g["nodes"], outs):
        args = [vals[a] for a in node["inputs"]]
        ref = oracle.run_node(node, args, mode="exact")
        if node["composite"] == "attention_tree":
            _, absum, score = D.attention_tree(node["attrs"], *args, magnitudes=True)
            d = node["attrs"]["head_dim"]
            bound = (2 * (d + 8) * E * score + 1000 * E + (U if dtype == "bf16" else 0)) * absum
        elif node["composite"] == "qk_norm_rotary":
            bound = np.full_like(ref, 2.0 ** -18 * np.abs(ref).max())
        elif node["composite"].startswith("logits"):
            bound = 6 * E * D.logits(node["composite"], node["attrs"], *args, magnitudes=True)[1]
            assert np.array_equal(y == -np.inf, ref == -np.inf)
            vals[node["name"]] = y
            y, ref = np.where(ref == -np.inf, 0, y), np.where(ref == -np.inf, 0, ref)
        else:
            bound = (2.0 ** -18 + (args[0].shape[1] + 8) * 2 * E) * (D.mxdense(args[0], args[1], magnitudes=True)[1] + 1 +
                                                                     (np.abs(args[3]) if len(args) == 4 else 0))
        _close(y, ref, bound, dtype)
        vals.setdefault(node["name"], y)


def test_verify_step_streams_graph_and_static_scratch():
    """The same bits on the current stream, on another one, replayed from a graph with eager work in between,
    captured by the caller, and with the intermediates in the static scratch."""
    import torch
    from paper_2105_03215_amd import capi, runtime
    wl = _step(batch=2, drafts=24, cached=600)
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        ins, outs = runtime.inputs_for(sg, wl.inputs, DEV), runtime.outputs_for(sg, DEV)
        sg.run(ins, outs)
        torch.cuda.synchronize()
        ref = [o.clone() for o in outs]
        s = torch.cuda.Stream(device=DEV)
        other = [torch.zeros_like(o) for o in outs]
        same = lambda: all(torch.equal(a, b) for a, b in zip(other, ref))  # noqa: E731
        s.wait_stream(torch.cuda.current_stream())
        sg.run(ins, other, s)
        s.synchronize()
        assert same()
        for o in other:
            o.zero_()
        torch.cuda.synchronize()
        sg.run_static(ins, other)
        torch.cuda.synchronize()
        assert same()
        first = ins[0].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sg.run(ins, other)
        sg.set_options(graph_replay=True)
        for k in range(6):
            ins[0].copy_(first if k % 2 == 0 else first * 0.5)
            torch.cuda.synchronize()
            if k < 4:
                sg.run(ins, other, s)
                s.synchronize()
            else:
                graph.replay()
                torch.cuda.synchronize()
            assert same() == (k % 2 == 0)
            torch.mm(torch.ones(64, 64, device=DEV), torch.ones(64, 64, device=DEV))
            torch.cuda.synchronize()
        sg.set_options(graph_replay=False, autotune=True)  # (nothing of the step is tuned; it must not mind)
        ins[0].copy_(first)
        sg.run(ins, other)
        torch.cuda.synchronize()
        assert same()


def test_verify_step_on_two_streams_at_once(monkeypatch):
    """A plan on two streams, and two engines on a stream each, have the bits of one alone."""
    import torch
    from paper_2105_03215_amd import capi, runtime
    wl = _step(batch=2, drafts=24, cached=600)
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        ref = runtime.run_once(sg, wl.inputs, DEV)
    monkeypatch.setenv("BYOC_STREAMS", "2")
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        got = runtime.run_once(sg, wl.inputs, DEV)
    assert all(np.array_equal(a, b) for a, b in zip(got, ref))
    monkeypatch.delenv("BYOC_STREAMS")
    with capi.Subgraph(wl.graph, wl.consts, device=0) as one, capi.Subgraph(wl.graph, wl.consts, device=0) as two:
        ins, outs = runtime.inputs_for(one, wl.inputs, DEV), [runtime.outputs_for(one, DEV) for _ in range(2)]
        streams = [torch.cuda.Stream(device=DEV) for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(3):
            for sg, o, s in zip((one, two), outs, streams):
                sg.run(ins, o, s)
        torch.cuda.synchronize()
        for o in outs:
            assert all(np.array_equal(runtime.to_host_f64(a), b) for a, b in zip(o, ref))


def test_verify_step_profile():
    from paper_2105_03215_amd import capi, runtime
    import torch
    wl = _step()
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        assert {l["kind"] for l in sg.launches()} == {"mxdense", "rotary", "attention", "logits"}
        ins, outs = runtime.inputs_for(sg, wl.inputs, DEV), runtime.outputs_for(sg, DEV)
        sg.profile_begin(2)
        for _ in range(2):
            sg.run(ins, outs)
        ms, runs = sg.profile_end()
        torch.cuda.synchronize()
        assert runs == 2 and all(t > 0 for t in ms)


def test_run_checks():
    """Buffers that the kernels address by their element are refused where they are not aligned to it."""
    import torch
    from paper_2105_03215_amd.capi import ByocError
    ins = _rules_case(2, 1, 64, 4, 0, "f32", "penalties")
    with _engine("logits_penalties", ins, list(ins), {"batch": 2}, "f32") as sg:
        from paper_2105_03215_amd import runtime
        bufs, out = runtime.inputs_for(sg, [a for a, _ in ins.values()], DEV), runtime.outputs_for(sg, DEV)
        sg.run(bufs, out)
        ptrs = [t.data_ptr() for t in bufs]
        for i, by in ((0, 4), (1, 2), (4, 2)):
            with pytest.raises(ByocError) as ei:
                sg.run(ptrs[:i] + [ptrs[i] + by] + ptrs[i + 1:], out)
            assert ei.value.status_name == "INVALID_ARG" and "input %d is not aligned" % i in str(ei.value)
        flat = torch.empty(2 * 64 + 4, device=DEV)
        with pytest.raises(ByocError):
            sg.run(bufs, [flat[1:129].view(2, 64)])
        # (strengths need no more than their own size)
        s = torch.empty(8, device=DEV)
        s[1:7] = bufs[4].reshape(-1)
        again = torch.empty_like(out[0])
        sg.run(bufs[:4] + [s[1:7].view(2, 3)], [again])
        torch.cuda.synchronize()
        assert torch.equal(again, out[0])
