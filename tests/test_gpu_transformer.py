"""Parity of the transformer-layer composites with their float64 definitions, at
the sizes, types, lengths and masks where they can go wrong.

Rounding bounds (u = 2^-8 for bf16, the largest relative error of its rounding;
e = 2^-24 for float32):
qdense     codes and their sums are exact (test values are bf16-representable, whose codes
           are those of the exact quotient); the scales, bias, residual and
           activation cost a few e of the terms' magnitudes, the bf16 output u of the result.
rotary     the reduced angle is 2^-25 turns off, sine and cosine 2^-22, the norm
           (D / 8 + 8) e: together under 2^-20 of |a| + |b| of the pair.
attention  a score is off by (D + 8) e sum |q||k| scale, which moves its weight by as much
           relatively, in numerator and denominator; the sums over n keys add (n + 64) e; in bf16
           each weight is rounded (u of sum p |v|) and the result again.
"""

import numpy as np
import pytest

import oracle
from oracle import transformer as T
from paper_2105_03215_amd import workloads
from paper_2105_03215_amd.workloads import to_bf16_values
from parity_util import announce, gate_end_to_end, rel_err

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U, E = 2.0 ** -8, 2.0 ** -24


def _engine(composite, ins, args, attrs, dtype, consts=()):
    """ins: name -> host array (int32 arrays are i32 inputs)."""
    from paper_2105_03215_amd import capi
    g = {"format": "byoc-subgraph", "version": 1,
         "inputs": [{"name": n, "shape": list(a.shape), "dtype": "i32" if a.dtype == np.int32 else dtype}
                    for n, a in ins.items()],
         "constants": [{"name": n, "index": i, "shape": list(a.shape), "dtype": "f32"}
                       for i, (n, a) in enumerate(consts)],
         "nodes": [{"name": "y", "composite": composite, "inputs": list(args), "attrs": attrs, "out_dtype": dtype}],
         "outputs": [{"name": "y", "dtype": dtype}]}
    return g, capi.Subgraph(g, [a for _, a in consts], device=0)


def _run(composite, ins, args, attrs, dtype, consts=()):
    from paper_2105_03215_amd import runtime
    _, sg = _engine(composite, ins, args, attrs, dtype, consts)
    try:
        out = runtime.run_once(sg, list(ins.values()), DEV)[0]
        again = runtime.run_once(sg, list(ins.values()), DEV)[0]
    finally:
        sg.close()
    assert np.array_equal(out, again, equal_nan=True)  # run to run identical
    return out


def _close(got, ref, bound, dtype):
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    ok = ~np.isnan(ref)
    slack = bound + (U * np.abs(ref) if dtype == "bf16" else 0.0)
    far = np.abs(got - ref)[ok] - slack[ok]
    assert far.size == 0 or far.max() <= 0, "%d of %d beyond the bound, worst by %.3g" % ((far > 0).sum(), far.size, far.max())


def _normal(rng, *shape, std=1.0):
    return to_bf16_values((rng.normal(size=shape) * std).astype(np.float32))


# ---- qdense ------------------------------------------------------------------

QDENSE = [
    # m, k, n, dtype, suffix
    (1, 64, 64, "bf16", "_bias_gelu"),
    (1, 8, 8, "bf16", ""),
    (1, 1, 1, "bf16", "_bias"),
    (1, 1, 1, "f32", "_bias"),
    (2, 1000, 24, "bf16", "_bias_add_relu"),
    (2, 512, 4104, "bf16", "_bias_gelu"),
    (8, 1000, 4096, "f32", "_bias"),
    (32, 384, 4096, "bf16", "_add"),
    (3, 129, 257, "bf16", "_bias"),
    (4, 4096, 96, "bf16", "_bias"),
    (5, 100, 1003, "f32", "_bias_add"),
    (13, 768, 300, "bf16", "_add_leaky"),
    (16, 1024, 128, "f32", "_relu6"),
    (17, 520, 72, "bf16", "_bias"),
    (33, 2000, 64, "f32", "_gelu"),
    (48, 640, 1000, "bf16", "_bias_gelu"),
    (63, 2048, 40, "bf16", "_bias"),
    (64, 96, 200, "bf16", "_bias_add"),
    (65, 384, 136, "bf16", ""),
    (130, 257, 131, "f32", "_bias"),
    (200, 8200, 64, "bf16", "_bias"),
    (300, 128, 520, "bf16", "_bias_add_gelu"),
    (1029, 136, 2056, "bf16", "_bias"),
    (2100, 256, 8000, "bf16", "_add"),
    (2100, 130, 2300, "f32", "_bias_add"),
]


@pytest.mark.parametrize("m, k, n, dtype, suffix", QDENSE)
def test_qdense(m, k, n, dtype, suffix):
    announce("qdense%s %dx%dx%d %s" % (suffix, m, k, n, dtype))
    r = np.random.default_rng(m * 1000003 + k * 101 + n)
    x, w = _normal(r, m, k), _normal(r, n, k, std=0.05)
    if m > 2:
        x[1] = 0
    if n > 2:
        w[2] = 0
    ins, args, consts = {"x": x}, ["x", "w"], [("w", w)]
    b, res = r.normal(size=n).astype(np.float32), _normal(r, m, n)
    if "_bias" in suffix:
        consts.append(("b", b))
        args.append("b")
    if "_add" in suffix:
        ins["r"] = res
        args.append("r")
    attrs = {"alpha": 0.2} if "leaky" in suffix else {}
    y = _run("qdense" + suffix, ins, args, attrs, dtype, consts)
    node = {"composite": "qdense" + suffix, "attrs": attrs, "out_dtype": dtype}
    ref = oracle.run_node(node, [x, w] + ([b] if "_bias" in suffix else []) + ([res] if "_add" in suffix else []),
                          mode="exact")
    terms = np.abs(T.qdense(x, w))
    terms = terms + (np.abs(b) if "_bias" in suffix else 0) + (np.abs(res) if "_add" in suffix else 0)
    # (GELU adds its own 2^-19 of the magnitude: its erfc is 1e-6 off at most)
    _close(y, ref, (2.0 ** -18 if "gelu" in suffix else 8 * E) * terms + 1e-37, dtype)


def test_qdense_f32_values_of_any_bits():
    """Values whose quotients fall next to the middle between two codes may take either code:
    one code of a row is one weight code times the scales."""
    r = np.random.default_rng(11)
    x, w = r.normal(size=(37, 300)).astype(np.float32), _normal(r, 50, 300)
    y = _run("qdense", {"x": x}, ["x", "w"], {}, "f32", [("w", w)])
    step = np.abs(x).max(axis=1)[:, None] / 127 * np.abs(w).max(axis=1)
    _close(y, T.qdense(x, w), step * 1.001, "f32")


@pytest.mark.parametrize("m, k, n, dtype, suffix", [
    (9, 1003, 4099, "bf16", "_bias_add_gelu"),
    (70, 515, 1001, "bf16", "_add"),
    (300, 2051, 301, "bf16", "_bias_add_relu"),
    (513, 130, 2305, "bf16", "_add"),
    (301, 515, 1003, "f32", "_bias_add"),
    (9, 7, 9, "bf16", "_add"),
])
def test_qdense_rows_at_any_address(m, k, n, dtype, suffix):
    """Rows of odd widths: their values start at any multiple of their own size."""
    test_qdense(m, k, n, dtype, suffix)


@pytest.mark.parametrize("m", [1, 9, 70])
def test_qdense_odd_rows(m):
    """Rows of zeros, of one value, with infinities and NaN, of the smallest and largest magnitudes."""
    r = np.random.default_rng(12)
    k, n = 200, 72
    w = _normal(r, n, k)
    rows = [np.zeros(k), np.full(k, -3.0), r.normal(size=k) * 1e-39, r.normal(size=k) * 2.0 ** -126,
            r.normal(size=k) * 2.0 ** 120, np.where(np.arange(k) == 77, np.inf, 1.0),
            np.where(np.arange(k) == 199, np.nan, 1.0), np.where(np.arange(k) == 0, -np.inf, 0.0)]
    for i, row in enumerate(rows):
        x = _normal(r, m, k)
        at = (3 * i) % m
        x[at] = to_bf16_values(row.astype(np.float32))
        with np.errstate(over="ignore"):
            y = _run("qdense", {"x": x}, ["x", "w"], {}, "bf16", [("w", w)])
            ref = T.qdense(x, w)
        # (sums of float32 denormals may flush: absolute slack of the smallest normal)
        _close(y, ref, 8 * E * np.abs(ref) + 2.0 ** -126, "bf16")


def test_qdense_odd_widths_between_layers():
    """Rows of a width that is no multiple of 8, as input, residual, between layers and twice an output."""
    from paper_2105_03215_amd import capi, runtime
    g = workloads.GraphBuilder("t", 97)
    x = g.input("x", [21, 77], "normal")
    r = g.input("r", [21, 131], "normal")
    h = g.qdense(x, 131, act="relu", residual=r)
    y = g.qdense(h, 53, act="gelu")
    z = g.add(h, r)
    for v in (y, h, y, z):
        g.output(v)
    wl = g.finish()
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        got = runtime.run_once(sg, wl.inputs, DEV)
    vals = {"x": wl.inputs[0], "r": wl.inputs[1]}
    by = {c["name"]: wl.consts[c["index"]] for c in wl.graph["constants"]}
    for node, v in zip(wl.graph["nodes"], (got[1], got[0], got[3])):
        ref = oracle.run_node(node, [vals.get(a, by.get(a)) for a in node["inputs"]], mode="exact")
        _close(v, ref, 2.0 ** -18 * (np.abs(ref) + 20), "bf16")
        vals[node["name"]] = v
    assert np.array_equal(got[0], got[2])


def test_qdense_rows_of_one_value_share_their_codes():
    """Two products of one value, and the graph that holds both, give what each gives alone."""
    from paper_2105_03215_amd import capi, runtime
    g = workloads.GraphBuilder("t", 99)
    x = g.input("x", [40, 96], "normal")
    a, b = g.qdense(x, 64, act="relu"), g.qdense(x, 200)
    g.output(a)
    g.output(b)
    wl = g.finish()
    sg = capi.Subgraph(wl.graph, wl.consts, device=0)
    try:
        names = [l["name"] for l in sg.launches()]
        ya, yb = runtime.run_once(sg, wl.inputs, DEV)
    finally:
        sg.close()
    assert sum(n == "quant_rows" for n in names) <= 1
    for y, ref in zip((ya, yb), oracle.run_graph(wl.graph, wl.consts, wl.inputs, mode="exact")):
        _close(y, ref, 8 * E * (np.abs(ref) + 1), "bf16")


# ---- rotary --------------------------------------------------------------------

ROTARY = [
    # m, heads, kv, d, rd, dtype, norm, layout, scaling, extra columns
    (1, 1, 0, 2, 2, "bf16", False, "half", None, 0),
    (1, 2, 1, 64, 64, "bf16", True, "half", None, 16),
    (4, 12, 12, 64, 64, "bf16", False, "half", None, 768),
    (5, 4, 2, 128, 128, "bf16", True, "half", "yarn", 0),
    (7, 3, 1, 80, 40, "bf16", True, "half", "linear", 8),
    (7, 3, 1, 80, 32, "f32", False, "interleaved", "ntk", 3),
    (9, 3, 0, 96, 96, "bf16", True, "interleaved", None, 0),
    (3, 2, 2, 6, 4, "bf16", True, "half", None, 1),
    (3, 5, 0, 10, 10, "bf16", False, "interleaved", None, 0),
    (11, 2, 2, 48, 24, "f32", True, "half", "yarn", 0),
    (6, 2, 1, 256, 256, "bf16", True, "half", "ntk", 0),
    (6, 1, 1, 512, 256, "f32", True, "interleaved", None, 0),
    (6, 1, 1, 512, 510, "bf16", False, "half", None, 0),
    (1030, 4, 1, 64, 64, "bf16", True, "half", None, 64),
    (2051, 3, 3, 32, 16, "bf16", False, "half", None, 0),
    (2051, 5, 1, 128, 128, "f32", True, "half", "linear", 0),
]
SCALINGS = {"linear": {"type": "linear", "factor": 4.0}, "ntk": {"type": "ntk", "factor": 2.5},
            "yarn": {"type": "yarn", "factor": 8.0, "original_length": 512}}


@pytest.mark.parametrize("m, heads, kv, d, rd, dtype, norm, layout, scaling, extra", ROTARY)
def test_rotary(m, heads, kv, d, rd, dtype, norm, layout, scaling, extra):
    announce("rotary m %d heads %d+%d d %d rd %d %s %s %s %s" % (m, heads, kv, d, rd, dtype, norm, layout, scaling))
    r = np.random.default_rng(m * 7 + d)
    x = _normal(r, m, (heads + kv) * d + extra)
    if m > 2:
        x[1] = 0
    pos = r.integers(0, 100000, m).astype(np.int32)
    pos[:min(m, 3)] = [0, 2 ** 31 - 1, -2 ** 31][:min(m, 3)]
    attrs = {"heads": heads, "kv_heads": kv, "head_dim": d, "rotary_dim": rd, "layout": layout, "base": 50000.0}
    if scaling:
        attrs["scaling"] = SCALINGS[scaling]
    ws = [(n, (1 + r.normal(size=d) * 0.2).astype(np.float32)) for n in ("wq", "wk")[:2 if kv else 1]] if norm else []
    y = _run("qk_norm_rotary" if norm else "rotary", {"x": x, "p": pos}, ["x"] + [n for n, _ in ws] + ["p"], attrs,
             dtype, ws)
    ref = T.rotary(attrs, x, pos, [w for _, w in ws] if norm else None)
    # |a| + |b| of each pair: the head's values normed, not turned
    xs = x[:, :(heads + kv) * d].astype(np.float64).reshape(m, heads + kv, d)
    if norm:
        xs = np.concatenate([T.qk_norm(xs[:, :heads], ws[0][1], 1e-6)] +
                            ([T.qk_norm(xs[:, heads:], ws[1][1], 1e-6)] if kv else []), axis=1)
    mag = np.abs(xs)
    a, b = (slice(0, rd, 2), slice(1, rd, 2)) if layout == "interleaved" else (slice(0, rd // 2), slice(rd // 2, rd))
    both = mag[..., a] + mag[..., b]
    mag[..., a] = mag[..., b] = both
    _close(y, ref, 2.0 ** -20 * 1.5 * mag.reshape(m, -1) + (d / 8 + 8) * E * mag.reshape(m, -1), dtype)


@pytest.mark.parametrize("m, heads, kv, d, rd, dtype, norm, layout, scaling, extra", [
    (5, 3, 2, 48, 24, "bf16", True, "half", None, 0),
    (1100, 2, 1, 80, 40, "bf16", False, "half", "linear", 5),
    (9, 2, 2, 80, 40, "f32", True, "half", "yarn", 8),
    (9, 3, 1, 8, 8, "bf16", True, "half", None, 0),
    (7, 2, 0, 56, 8, "f32", False, "half", None, 4),
    (7, 2, 1, 40, 20, "bf16", True, "half", None, 0),
])
def test_rotary_halves_of_no_whole_chunks(m, heads, kv, d, rd, dtype, norm, layout, scaling, extra):
    """Pairs whose two columns lie in 16-byte chunks at different places."""
    test_rotary(m, heads, kv, d, rd, dtype, norm, layout, scaling, extra)


def test_rotary_padding_columns_are_zero():
    """Heads that do not fill a multiple of 8 columns feed a dense layer, which reads the padding."""
    from paper_2105_03215_amd import capi, runtime
    g = workloads.GraphBuilder("t", 98)
    x = g.input("x", [9, 40], "normal")
    p = g.index_input("p", np.arange(9))
    y = g.dense(g.rotary(x, p, 3, 0, 6), 16)
    g.output(y)
    wl = g.finish()
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        import torch
        # every arena byte a NaN first
        ins, outs = runtime.inputs_for(sg, wl.inputs, DEV), runtime.outputs_for(sg, DEV)
        nan = [torch.full_like(t, float("nan")) if t.is_floating_point() else t for t in ins]
        sg.run(nan, outs)
        sg.run(ins, outs)
        torch.cuda.synchronize()
        got = runtime.to_host_f64(outs[0])
    ref = oracle.run_graph(wl.graph, wl.consts, wl.inputs)[0]
    assert rel_err(got, ref) <= 1e-2


# ---- attention -------------------------------------------------------------------

ATTENTION = [
    # batch, q_len, k_len, heads, kv, d, dtype, causal, lengths
    (1, 1, 1, 1, 1, 8, "bf16", False, None),
    (1, 1, 1, 1, 1, 8, "f32", True, None),
    (2, 1, 31, 2, 2, 64, "bf16", False, [31, 7]),
    (2, 1, 33, 4, 1, 64, "bf16", False, [33, 0]),
    (3, 1, 700, 8, 2, 128, "bf16", False, [700, 1, 129]),
    (3, 1, 700, 8, 2, 128, "f32", False, [700, 1, 129]),
    (1, 1, 5000, 4, 4, 80, "bf16", False, None),
    (1, 3, 1100, 16, 1, 40, "bf16", True, [1055]),
    (2, 5, 3, 4, 2, 72, "bf16", True, None),        # more queries than keys: the first see none
    (2, 5, 9, 4, 2, 72, "f32", True, [9, 3]),
    (2, 64, 64, 2, 2, 64, "bf16", True, None),
    (2, 65, 64, 2, 1, 64, "bf16", False, [64, 63]),
    (1, 130, 257, 3, 3, 96, "bf16", False, [200]),
    (1, 130, 257, 3, 3, 96, "f32", True, None),
    (2, 128, 128, 4, 2, 128, "bf16", True, [128, 100]),
    (1, 300, 513, 2, 1, 128, "bf16", True, None),
    (1, 257, 320, 2, 2, 64, "bf16", False, [320]),
    (1, 70, 90, 2, 1, 256, "bf16", False, None),
    (1, 40, 90, 2, 2, 256, "f32", True, None),
    (2, 33, 100, 1, 1, 24, "bf16", False, [100, -5]),   # (lengths outside [0, k_len] are taken as its ends)
    (2, 2, 100, 1, 1, 32, "bf16", False, [101, 2 ** 31 - 1]),
    (4, 200, 200, 4, 4, 64, "bf16", False, [0, 1, 199, 200]),
]


def _attention(batch, q_len, k_len, heads, kv, d, dtype, causal, lengths, seed=0, std=1.0, spoil=False, scale=None):
    r = np.random.default_rng(seed + batch * 31 + q_len * 7 + k_len + d)
    q = _normal(r, batch * q_len, 8 + heads * d, std=std)
    kvt = _normal(r, batch * k_len, 8 + 2 * kv * d)
    ins, args = {"q": q, "kv": kvt}, ["q", "kv", "kv"]
    attrs = {"batch": batch, "heads": heads, "kv_heads": kv, "head_dim": d, "causal": causal, "q_col": 8, "k_col": 8,
             "v_col": 8 + kv * d}
    if scale:
        attrs["scale"] = scale
    if lengths is not None:
        ins["n"] = np.array(lengths, np.int64).astype(np.int32)
        args.append("n")
        if spoil:  # what stands past the lengths must not be seen
            rows = kvt.reshape(batch, k_len, -1)
            for i, n in enumerate(lengths):
                rows[i, min(max(n, 0), k_len):] = [np.nan, np.inf, -np.inf][i % 3]
    y = _run("attention" if lengths is None else "attention_lengths", ins, args, attrs, dtype)
    ref, absum, score = T.attention(attrs, q, kvt, kvt, lengths, magnitudes=True)
    delta = (d + 8) * E * score
    bound = (2 * delta + (k_len + 64) * E + (U if dtype == "bf16" else 0)) * absum
    return y, ref, bound


@pytest.mark.parametrize("batch, q_len, k_len, heads, kv, d, dtype, causal, lengths", ATTENTION)
def test_attention(batch, q_len, k_len, heads, kv, d, dtype, causal, lengths):
    announce("attention b %d q %d k %d heads %d/%d d %d %s causal %s lengths %s" % (
        batch, q_len, k_len, heads, kv, d, dtype, causal, lengths))
    y, ref, bound = _attention(batch, q_len, k_len, heads, kv, d, dtype, causal, lengths, spoil=True)
    _close(y, ref, bound, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len, k_len", [(1, 900), (150, 300)])
def test_attention_sharp_scores(q_len, k_len, dtype):
    """Scores far apart: almost every weight is zero, the maximum moves along the keys."""
    y, ref, bound = _attention(1, q_len, k_len, 2, 1, 64, dtype, False, None, seed=3, std=30.0)
    _close(y, ref, bound, dtype)
    y, ref, bound = _attention(1, q_len, k_len, 2, 1, 64, dtype, True, None, seed=4, scale=1e-3)
    _close(y, ref, bound, dtype)


@pytest.mark.parametrize("q_len", [1, 200])
def test_attention_growing_scores(q_len):
    """Every tile of keys holds a new maximum: the sums are rescaled each time."""
    n, d = 640, 64
    k = np.zeros((n, 2 * d), np.float32)
    k[:, 0] = np.arange(n) / 8.0
    k[:, d:] = to_bf16_values(np.random.default_rng(1).normal(size=(n, d)).astype(np.float32))
    k[:, 0] = to_bf16_values(k[:, 0])
    q = np.zeros((q_len, d), np.float32)
    q[:, 0] = 8.0
    for sign in (1, -1):
        ins = {"q": sign * q, "kv": k}
        attrs = {"batch": 1, "heads": 1, "head_dim": d, "v_col": d}
        y = _run("attention", ins, ["q", "kv", "kv"], attrs, "bf16")
        ref, absum, score = T.attention(attrs, sign * q, k, k, None, magnitudes=True)
        _close(y, ref, (2 * (d + 8) * E * score + (n + 64) * E + U) * absum, "bf16")


@pytest.mark.parametrize("q_len", [1, 160])
def test_attention_infinities_and_nan_in_seen_places(q_len):
    """They come out where the definition has them, and nowhere else."""
    n, d = 200, 64
    r = np.random.default_rng(5)
    q, kv = _normal(r, 2 * q_len, d), _normal(r, 2 * n, 2 * d)
    kv[150, d + 3] = np.nan      # a value: its column, in batch 0
    kv[n + 7, 5] = np.nan        # a key: every column of batch 1
    attrs = {"batch": 2, "heads": 1, "head_dim": d, "v_col": d}
    y = _run("attention", {"q": q, "kv": kv}, ["q", "kv", "kv"], attrs, "bf16")
    assert np.isnan(y[:q_len, 3]).all() and not np.isnan(np.delete(y[:q_len], 3, axis=1)).any()
    assert np.isnan(y[q_len:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len, k_len, d", [(8, 50, 64), (100, 100, 64), (100, 100, 128), (300, 300, 32), (70, 70, 256)])
def test_attention_causal_hides_infinities_and_nan(q_len, k_len, d, dtype):
    """A key that a row does not see cannot reach it, though its tile holds rows that see it."""
    r = np.random.default_rng(7)
    h, kv = 4, 2
    q, k, v = _normal(r, q_len, h * d), _normal(r, k_len, kv * d), _normal(r, k_len, kv * d)
    v[k_len - 3, 1] = np.nan
    v[k_len - 5, d + 2] = np.inf
    v[k_len - 4, 7] = -np.inf
    k[k_len - 1, d:] = np.nan
    attrs = {"batch": 1, "heads": h, "kv_heads": kv, "head_dim": d, "causal": True}
    y = _run("attention", {"q": q, "k": k, "v": v}, ["q", "k", "v"], attrs, dtype)
    with np.errstate(invalid="ignore"):
        ref, absum, score = T.attention(attrs, q, k, v, None, magnitudes=True)
    assert np.array_equal(np.isnan(y), np.isnan(ref)) and np.isnan(ref).any() and not np.isnan(ref).all()
    inf = np.isinf(ref)
    assert inf.any() and np.array_equal(y[inf], ref[inf])
    fine = np.isfinite(ref)
    bound = (2 * (d + 8) * E * score + (k_len + 64) * E + (U if dtype == "bf16" else 0)) * absum
    _close(y[fine], ref[fine], bound[fine], dtype)


def test_attention_separate_and_shared_inputs_agree():
    r = np.random.default_rng(6)
    b, lq, lk, h, d = 2, 40, 70, 2, 64
    q, k, v = _normal(r, b * lq, h * d), _normal(r, b * lk, h * d), _normal(r, b * lk, h * d)
    attrs = {"batch": b, "heads": h, "head_dim": d}
    a = _run("attention", {"q": q, "k": k, "v": v}, ["q", "k", "v"], attrs, "bf16")
    c = _run("attention", {"q": q, "kv": np.concatenate([k, v], axis=1)}, ["q", "kv", "kv"],
             dict(attrs, v_col=h * d), "bf16")
    assert np.array_equal(a, c)


# Key axes split over workgroups: sequences of one length and of different ones, empty ones among them,
# more sequences than a wave has lanes, chunks that some rows see nothing of, joins of few and of many chunks.
ATTENTION_SPLIT = [
    (16, 1, 3000, 4, 4, 64, "bf16", False, None),
    (1, 1, 9000, 16, 1, 128, "bf16", False, None),
    (1, 1, 9001, 2, 1, 256, "bf16", False, [8999]),
    (5, 7, 4100, 2, 1, 40, "f32", True, [4100, 0, 3, 1500, 2222]),
    (12, 1, 2000, 2, 2, 128, "bf16", False, [2000, 1, 0, 999, 1024, 1025, 31, 33, 0, 1999, 500, 1700]),
    (64, 1, 800, 1, 1, 64, "bf16", False, [(37 * i) % 801 for i in range(64)]),
    (70, 1, 500, 1, 1, 32, "bf16", False, [(61 * i) % 501 for i in range(70)]),
    (70, 1, 1700, 1, 1, 64, "bf16", False, [(211 * i) % 1701 for i in range(70)]),
    (67, 33, 4100, 1, 1, 32, "bf16", False, [(611 * i) % 4101 for i in range(67)]),
    (33, 34, 4100, 1, 1, 64, "bf16", False, [(711 * i) % 4101 for i in range(33)]),
    (3, 50, 3000, 2, 2, 64, "bf16", True, None),
    (2, 45, 2600, 1, 1, 128, "bf16", True, [2600, 40]),
]


@pytest.mark.parametrize("batch, q_len, k_len, heads, kv, d, dtype, causal, lengths", ATTENTION_SPLIT)
def test_attention_split_keys(batch, q_len, k_len, heads, kv, d, dtype, causal, lengths):
    announce("attention split b %d q %d k %d heads %d/%d d %d %s" % (batch, q_len, k_len, heads, kv, d, dtype))
    y, ref, bound = _attention(batch, q_len, k_len, heads, kv, d, dtype, causal, lengths, seed=8, spoil=lengths is not None)
    _close(y, ref, bound, dtype)


@pytest.mark.parametrize("batch, q_len, k_len, heads, kv, d, causal, lengths", [
    (130, 33, 1, 1, 1, 8, False, None),
    (64, 40, 100, 2, 2, 64, True, [(29 * i) % 101 for i in range(64)]),  # (rows that see no key, tiles that end inside)
    (16, 100, 128, 8, 8, 40, True, None),
    (64, 130, 33, 1, 1, 64, False, [(5 * i) % 34 for i in range(64)]),
    (32, 40, 140, 8, 8, 128, False, [140 - 4 * i for i in range(32)]),
    (256, 36, 45, 1, 1, 256, True, None),
    (8, 65, 330, 32, 32, 72, True, [330, 0, 1, 64, 65, 66, 200, 329]),
    (43, 200, 35, 6, 1, 200, False, None),
])
def test_attention_f32_many_rows(batch, q_len, k_len, heads, kv, d, causal, lengths):
    announce("attention f32 b %d q %d k %d heads %d/%d d %d" % (batch, q_len, k_len, heads, kv, d))
    y, ref, bound = _attention(batch, q_len, k_len, heads, kv, d, "f32", causal, lengths, seed=9, spoil=lengths is not None)
    _close(y, ref, bound, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 32, 40, 72, 88, 96, 104, 136, 192, 200])
def test_attention_head_sizes(d, dtype):
    """Heads that end inside the columns that are multiplied, for few rows and for many, masked and not."""
    for q_len, causal in ((1, False), (45, True), (150, False)):
        y, ref, bound = _attention(2, q_len, 170, 2, 1, d, dtype, causal, [170, 133], seed=d, spoil=True)
        _close(y, ref, bound, dtype)


# ---- buffers, streams, graphs -------------------------------------------------------

def test_misaligned_buffers_are_refused():
    import torch
    from paper_2105_03215_amd.capi import ByocError
    x, p = np.zeros((4, 64), np.float32), np.zeros(4, np.int32)
    _, sg = _engine("rotary", {"x": x, "p": p}, ["x", "p"], {"heads": 1, "head_dim": 64}, "bf16")
    with sg:
        flat = torch.zeros(4 * 64 + 8, dtype=torch.bfloat16, device=DEV)
        pos, out = torch.zeros(4, dtype=torch.int32, device=DEV), torch.empty(4, 64, dtype=torch.bfloat16, device=DEV)
        sg.run([flat[:256].view(4, 64), pos], [out])
        with pytest.raises(ByocError) as ei:
            sg.run([flat[1:257].view(4, 64), pos], [out])
        assert ei.value.status_name == "INVALID_ARG" and "input 0 is not aligned to 16" in str(ei.value)
        with pytest.raises(ByocError) as ei:
            sg.run([flat[:256].view(4, 64), pos], [flat[4:260].view(4, 64)])
        assert "output 0 is not aligned" in str(ei.value)
        with pytest.raises(ByocError):
            sg.run([flat[:256].view(4, 64), pos.long()], [out])
        torch.cuda.synchronize()


def _layer(**kw):
    kw = dict(dict(batch=3, tokens=17, encoder_tokens=37, hidden=256, heads=4, kv_heads=2, ffn=320), **kw)
    return workloads.build("decoder_layer", **kw)


@pytest.mark.parametrize("kw", [dict(), dict(tokens=1, start=900), dict(batch=1, tokens=130, encoder_tokens=1)])
def test_decoder_layer_teacher_forced(kw):
    """The composites of a layer run together, each as an output of the engine, against the
    oracle on the engine's own inputs of that node: one rounding of bf16 each, and of the weights in attention."""
    from paper_2105_03215_amd import capi, runtime
    wl = _layer(**kw)
    g = dict(wl.graph, outputs=[{"name": n["name"], "dtype": "bf16"} for n in wl.graph["nodes"]])
    with capi.Subgraph(g, wl.consts, device=0) as sg:
        outs = runtime.run_once(sg, wl.inputs, DEV)
    vals = {d["name"]: np.asarray(a, np.float64) for d, a in zip(g["inputs"], wl.inputs)}
    for c in g["constants"]:
        vals[c["name"]] = np.asarray(wl.consts[c["index"]], np.float64)
    for node, y in zip(g["nodes"], outs):
        args = [vals[a] for a in node["inputs"]]
        ref = oracle.run_node(node, args, mode="exact")
        if node["composite"].startswith("attention"):
            _, absum, score = T.attention(node["attrs"], *args, magnitudes=True)
            d = node["attrs"]["head_dim"]
            bound = (2 * (d + 8) * E * score + 200 * E + U) * absum
        elif node["composite"] == "qk_norm_rotary":
            bound = np.full_like(ref, 2.0 ** -18 * np.abs(ref).max())
        else:
            bound = 2.0 ** -18 * (np.abs(T.qdense(args[0], args[1])) + 1 + (np.abs(args[3]) if len(args) == 4 else 0))
        _close(y, ref, bound, "bf16")
        vals[node["name"]] = y


def test_decoder_layer_end_to_end():
    from paper_2105_03215_amd import capi, runtime
    wl = _layer()
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        got = runtime.run_once(sg, wl.inputs, DEV)[0]
    ref = oracle.run_graph(wl.graph, wl.consts, wl.inputs)[0]
    exact = oracle.run_graph(wl.graph, wl.consts, wl.inputs, mode="exact")[0]
    gate_end_to_end(rel_err(got, ref), rel_err(ref, exact), "decoder layer")


def test_decoder_layer_streams_graph_and_static_scratch():
    """The same bits on the current stream, on another one, replayed from a graph with eager
    work in between, and with the intermediates in the static scratch."""
    import torch
    from paper_2105_03215_amd import capi, runtime
    wl = _layer(batch=2, tokens=40, encoder_tokens=300)
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        ins, outs = runtime.inputs_for(sg, wl.inputs, DEV), runtime.outputs_for(sg, DEV)
        sg.run(ins, outs)
        torch.cuda.synchronize()
        ref = outs[0].clone()
        s = torch.cuda.Stream(device=DEV)
        other = [torch.zeros_like(outs[0])]
        s.wait_stream(torch.cuda.current_stream())
        sg.run(ins, other, s)
        s.synchronize()
        assert torch.equal(other[0], ref)
        other[0].zero_()
        torch.cuda.synchronize()
        sg.run_static(ins, other)
        torch.cuda.synchronize()
        assert torch.equal(other[0], ref)
        sg.set_options(graph_replay=True)
        first = ins[0].clone()
        for k in range(4):
            ins[0].copy_(first if k % 2 == 0 else first * 0.5)
            torch.cuda.synchronize()
            sg.run(ins, other, s)
            s.synchronize()
            assert torch.equal(other[0], ref) == (k % 2 == 0)
            torch.mm(torch.ones(64, 64, device=DEV), torch.ones(64, 64, device=DEV))
            torch.cuda.synchronize()
        sg.set_options(graph_replay=False, autotune=True)  # (nothing of the layer is tuned; it must not mind)
        ins[0].copy_(first)
        sg.run(ins, other)
        torch.cuda.synchronize()
        assert torch.equal(other[0], ref)


def test_decoder_layer_profile():
    from paper_2105_03215_amd import capi, runtime
    import torch
    wl = _layer()
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        kinds = {l["kind"] for l in sg.launches()}
        assert kinds == {"qdense", "rotary", "attention"}
        ins, outs = runtime.inputs_for(sg, wl.inputs, DEV), runtime.outputs_for(sg, DEV)
        sg.profile_begin(2)
        for _ in range(2):
            sg.run(ins, outs)
        ms, runs = sg.profile_end()
        torch.cuda.synchronize()
        assert runs == 2 and all(t > 0 for t in ms)
