"""The transformer-layer composites at the edges of their ranges: magnitudes near the ends of float32, infinities
and NaN without a loss of speed, every product tile, and what a plan shares, pads and overlaps.

Rounding bounds as in test_gpu_transformer (u = 2^-8, e = 2^-24), and: an angle in turns is off by 2^-24 where a
position is near 2^31 (53 bits of turns per position times 31 of position) and by 2^-26 from its rounding to float32.
"""

import decimal

import numpy as np
import pytest

import oracle
from oracle import transformer as T
from paper_2105_03215_amd import workloads
from paper_2105_03215_amd.workloads import to_bf16_values
from parity_util import announce, bf16_ulp
from test_gpu_transformer import DEV, E, U, _close, _engine, _layer, _normal, _run

pytestmark = pytest.mark.gpu


# ---- rotary --------------------------------------------------------------------

@pytest.mark.parametrize("heads, kv, d, rd, layout, dtype", [
    (2, 1, 128, 128, "half", "bf16"),
    (2, 1, 128, 128, "half", "f32"),
    (1, 0, 64, 64, "interleaved", "bf16"),
    (3, 1, 80, 40, "half", "bf16"),
    (2, 2, 6, 4, "half", "bf16"),
    (1, 1, 512, 510, "interleaved", "f32"),
])
def test_norm_of_large_heads(heads, kv, d, rd, layout, dtype):
    """Heads whose squares leave float32 have a norm all the same; one that holds an infinity has none, and its other
    columns are zero, as a number over infinity is."""
    announce("norm of large heads %d+%d d %d rd %d %s %s" % (heads, kv, d, rd, layout, dtype))
    r = np.random.default_rng(d + rd)
    powers = [0, 40, 58, 60, 62, 64, 66, 90, 124]
    x = _normal(r, len(powers) + 2, (heads + kv) * d)
    x[:len(powers)] = to_bf16_values((x[:len(powers)] * np.exp2(np.array(powers))[:, None]).astype(np.float32))
    x[-2, 1] = 2.0 ** 126       # one value above the others of its head
    x[-1, 0] = np.inf
    pos = np.arange(len(x)).astype(np.int32)
    attrs = {"heads": heads, "kv_heads": kv, "head_dim": d, "rotary_dim": rd, "layout": layout}
    ws = [(n, (1 + r.normal(size=d) * 0.2).astype(np.float32)) for n in ("wq", "wk")[:2 if kv else 1]]
    y = _run("qk_norm_rotary", {"x": x, "p": pos}, ["x"] + [n for n, _ in ws] + ["p"], attrs, dtype, ws)
    with np.errstate(invalid="ignore"):
        ref = T.rotary(attrs, x, pos, [w for _, w in ws])
    # a normed value is sqrt(D) at most, and a pair is two (weights below 2)
    _close(y, ref, np.full_like(ref, (2.0 ** -20 * 1.5 + (d / 8 + 8) * E) * 4 * d ** 0.5), dtype)
    assert (np.abs(ref[:len(powers)]).max(axis=1) > 0.5).all()


@pytest.mark.parametrize("d, dtype", [(64, "bf16"), (10, "bf16"), (64, "f32")])
def test_norm_of_zeros_with_the_smallest_eps(d, dtype):
    """A head of zeros is zero for every positive eps, also one below float32."""
    x = _normal(np.random.default_rng(2), 5, 2 * d)
    x[1], x[3, d:] = 0, 0
    w = np.ones(d, np.float32)
    attrs = {"heads": 2, "head_dim": d, "eps": 1e-60}
    y = _run("qk_norm_rotary", {"x": x, "p": np.arange(5, dtype=np.int32)}, ["x", "w", "p"], attrs, dtype, [("w", w)])
    ref = T.rotary(attrs, x, np.arange(5), [w])
    _close(y, ref, np.full_like(ref, (2.0 ** -20 * 1.5 + (d / 8 + 8) * E) * 4 * d ** 0.5), dtype)


def test_rotary_angles_of_the_farthest_positions():
    """Sines and cosines at both ends of 32 bits, against 60 digits."""
    d = 64
    pos = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, -(2 ** 29) - 1, 123456789], np.int32)
    x = np.zeros((len(pos), d), np.float32)
    x[:, :d // 2] = 1.0  # (a, b) = (1, 0) of every pair: its cosine and sine come out
    y = _run("rotary", {"x": x, "p": pos}, ["x", "p"], {"heads": 1, "head_dim": d}, "f32")
    with decimal.localcontext() as c:
        c.prec = 60
        two_pi = 2 * decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
        ref = np.zeros_like(y)
        for i in range(d // 2):
            theta = decimal.Decimal(10000) ** (decimal.Decimal(-2 * i) / d)
            for m, p in enumerate(pos):
                turns = int(p) * theta / two_pi
                angle = float((turns - turns.to_integral_value()) * two_pi)
                ref[m, i], ref[m, i + d // 2] = np.cos(angle), np.sin(angle)
    _close(y, ref, np.full_like(ref, 2.0 ** -20), "f32")


def test_rotary_padding_columns_written_over_nan():
    """The padding columns of a rotation inside a plan are zeros, whatever the memory held: the intermediates stand in
    the static scratch, where an engine of NaN values ran before."""
    import torch
    from paper_2105_03215_amd import capi, runtime
    p = workloads.GraphBuilder("poison", 96)
    p.output(p.qdense(p.qdense(p.input("x", [8, 64], "normal"), 512), 64))  # (qdense keeps a NaN; one launch each)
    pw = p.finish()
    g = workloads.GraphBuilder("t", 98)
    x = g.input("x", [9, 40], "normal")
    g.output(g.dense(g.rotary(x, g.index_input("p", np.arange(9)), 3, 0, 6), 16))
    wl = g.finish()
    with capi.Subgraph(pw.graph, pw.consts, device=0) as poison, capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        # 18 columns padded to 24 of 9 rows stand where the poison's 8 x 512 values stood
        assert sg.stats()["arena_bytes"] >= 9 * 24 * 2 and poison.stats()["arena_bytes"] >= 8 * 512 * 2
        pin, pout = runtime.inputs_for(poison, pw.inputs, DEV), runtime.outputs_for(poison, DEV)
        pin[0].fill_(float("nan"))
        ins, outs = runtime.inputs_for(sg, wl.inputs, DEV), runtime.outputs_for(sg, DEV)
        poison.run_static(pin, pout)
        sg.run_static(ins, outs)
        torch.cuda.synchronize()
        assert torch.isnan(pout[0]).all()
        got = runtime.to_host_f64(outs[0])
    ref = oracle.run_graph(wl.graph, wl.consts, wl.inputs)[0]
    assert np.isfinite(got).all() and np.abs(got - ref).max() <= 1e-2 * (1 + np.abs(ref).max())


# ---- qdense ----------------------------------------------------------------------

@pytest.mark.parametrize("m", [1, 9, 70])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_qdense_scales_whose_product_leaves_float32(m, dtype):
    """Sums times scales that are numbers, though the product of the two scales is below the normal range or above all
    of it."""
    r = np.random.default_rng(21)
    k, n = 8192, 40
    x, w = np.abs(_normal(r, m, k, std=2.0 ** -66)), np.abs(_normal(r, n, k, std=2.0 ** -66))
    y = _run("qdense", {"x": x}, ["x", "w"], {}, dtype, [("w", w)])
    ref = T.qdense(x, w)
    assert np.abs(ref).min() > 2.0 ** -122  # (a_m / 127) (b_n / 127) is about 2^-142
    _close(y, ref, 8 * E * np.abs(ref), dtype)
    # a sum of zero between rows whose scales multiply to more than float32 holds
    x, w = np.full((m, 2), 2.0 ** 110, np.float32), np.full((n, 2), 2.0 ** 40, np.float32)
    x[:, 1] *= -1
    b = r.normal(size=n).astype(np.float32)
    y = _run("qdense_bias", {"x": x}, ["x", "w", "b"], {}, dtype, [("w", w), ("b", b)])
    _close(y, np.broadcast_to(b, (m, n)).astype(np.float64), np.full((m, n), 4 * E), dtype)


TILES = ["256x256_s2", "256x128_s3", "128x128_s3", "128x128_s2", "128x64_s3", "64x64_s4", "32x32_s8"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tile", range(len(TILES)))
@pytest.mark.parametrize("m, k, n, suffix", [
    (70, 100, 300, "_bias_add"),          # one stage of 128 codes, in any ring; a part of a tile either way
    (300, 390, 525, "_bias_add_gelu"),    # rows and channels past the largest tile
    (517, 1283, 264, "_add_leaky"),       # 11 stages
    (1100, 257, 1030, "_bias_relu"),      # more tiles than XCDs, in bands of rows
])
def test_qdense_every_tile(m, k, n, suffix, tile, dtype, monkeypatch):
    announce("qdense%s %dx%dx%d %s on %s" % (suffix, m, k, n, dtype, TILES[tile]))
    r = np.random.default_rng(m + k + n)
    x, w = _normal(r, m, k), _normal(r, n, k, std=0.05)
    b, res = r.normal(size=n).astype(np.float32), _normal(r, m, n)
    ins, args, consts = {"x": x}, ["x", "w"], [("w", w)]
    if "_bias" in suffix:
        consts.append(("b", b))
        args.append("b")
    if "_add" in suffix:
        ins["r"] = res
        args.append("r")
    attrs = {"alpha": 0.2} if "leaky" in suffix else {}
    monkeypatch.setenv("BYOC_QDENSE_TILE", str(tile))
    _, sg = _engine("qdense" + suffix, ins, args, attrs, dtype, consts)
    with sg:
        assert [l["name"] for l in sg.launches()] == ["quant_rows", "qdense_" + TILES[tile]]
    y = _run("qdense" + suffix, ins, args, attrs, dtype, consts)
    ref = oracle.run_node({"composite": "qdense" + suffix, "attrs": attrs, "out_dtype": dtype},
                          [x, w] + ([b] if "_bias" in suffix else []) + ([res] if "_add" in suffix else []), mode="exact")
    terms = np.abs(T.qdense(x, w)) + (np.abs(b) if "_bias" in suffix else 0) + (np.abs(res) if "_add" in suffix else 0)
    _close(y, ref, (2.0 ** -18 if "gelu" in suffix else 8 * E) * terms + 1e-37, dtype)


@pytest.mark.parametrize("m, k, n, name", [
    (901, 100, 8201, "256x256_s2"),
    (513, 2051, 8200, "256x128_s3"),
    (200, 1000, 8200, "128x128_s3"),
    (1029, 100, 4100, "128x128_s2"),
    (200, 129, 8200, "128x64_s3"),
    (33, 129, 8200, "64x64_s4"),
    (70, 300, 130, "32x32_s8"),
])
def test_qdense_tiles_that_the_sizes_choose(m, k, n, name):
    """The tile of least modelled time, whole and at its remainders."""
    announce("qdense %dx%dx%d on %s" % (m, k, n, name))
    r = np.random.default_rng(m + k + n)
    x, w, res = _normal(r, m, k), _normal(r, n, k, std=0.05), _normal(r, m, n)
    _, sg = _engine("qdense_add", {"x": x, "r": res}, ["x", "w", "r"], {}, "bf16", [("w", w)])
    with sg:
        assert [l["name"] for l in sg.launches()] == ["quant_rows", "qdense_" + name]
    y = _run("qdense_add", {"x": x, "r": res}, ["x", "w", "r"], {}, "bf16", [("w", w)])
    ref = T.qdense(x, w)
    _close(y, ref + res, 8 * E * (np.abs(ref) + np.abs(res)) + 1e-37, "bf16")


def test_qdense_gelu_of_bf16_far_below_zero():
    """A GELU in bf16 down to -9 is off by its rounding, half a step of bf16 there, and 2^-16 for the short form."""
    n = 4096
    b = np.linspace(-9, 9, n).astype(np.float32)
    for m in (1, 20, 40):  # rows of zeros: the bias alone
        x = np.zeros((m, 64), np.float32)
        y = _run("qdense_bias_gelu", {"x": x}, ["x", "w", "b"], {}, "bf16", [("w", np.ones((n, 64), np.float32)), ("b", b)])
        ref = np.broadcast_to(oracle.run_node({"composite": "dense_bias_gelu", "out_dtype": "f32"},
                                              [np.zeros((1, 1)), np.zeros((n, 1)), b], mode="exact"), (m, n))
        # (the steps of a value that the short form may have moved past a power of two)
        assert (np.abs(y - ref) <= 0.5 * bf16_ulp(ref * (1 + 2.0 ** -16)) + 2.0 ** -16 * np.abs(ref)).all()


def test_qdense_rows_are_quantized_once_for_all_their_products():
    """One quantization of a value that two products read, and the bits that each product has alone."""
    from paper_2105_03215_amd import capi, runtime
    g = workloads.GraphBuilder("t", 99)
    x = g.input("x", [40, 96], "normal")
    g.output(g.qdense(x, 64, act="relu"))
    g.output(g.qdense(x, 200))
    wl = g.finish()
    with capi.Subgraph(wl.graph, wl.consts, device=0) as sg:
        assert [l["name"] for l in sg.launches()].count("quant_rows") == 1
        both = runtime.run_once(sg, wl.inputs, DEV)
    for node, y in zip(wl.graph["nodes"], both):
        names = set(node["inputs"])
        consts = [c for c in wl.graph["constants"] if c["name"] in names]
        alone = dict(wl.graph, nodes=[node], outputs=[{"name": node["name"], "dtype": "bf16"}],
                     constants=[dict(c, index=i) for i, c in enumerate(consts)])
        with capi.Subgraph(alone, [wl.consts[c["index"]] for c in consts], device=0) as sg:
            assert [l["name"] for l in sg.launches()].count("quant_rows") == 1
            assert np.array_equal(runtime.run_once(sg, wl.inputs, DEV)[0], y)


# ---- attention -------------------------------------------------------------------

@pytest.mark.parametrize("k_len, d, group", [(64, 64, 1), (200, 128, 4), (70, 256, 2), (600, 64, 8)])
def test_attention_weights_of_few_rows_are_not_rounded_to_bf16(k_len, d, group):
    """Values that cancel leave the error of the weights alone: where few rows share the keys 2^-16 of each, two
    roundings to bf16 one after the other."""
    announce("attention weights k %d d %d group %d" % (k_len, d, group))
    r = np.random.default_rng(k_len + d)
    # (scores near each other, so that their own rounding stays below that of the weights)
    q, k = np.repeat(_normal(r, 1, d, std=0.02), group, axis=0).reshape(1, -1), _normal(r, k_len, d)
    v = r.normal(size=(k_len, d))
    s = k.astype(np.float64) @ q[0, :d].astype(np.float64) / d ** 0.5
    p = np.exp(s - s.max())
    p /= p.sum()
    big = np.argmax(p)
    v[big] = 0
    v[big] = -(p @ v) / p[big]
    v = to_bf16_values(v.astype(np.float32))
    attrs = {"batch": 1, "heads": group, "kv_heads": 1, "head_dim": d}
    y = _run("attention", {"q": q, "k": k, "v": v}, ["q", "k", "v"], attrs, "bf16")
    ref, absum, score = T.attention(attrs, q, k, v, None, magnitudes=True)
    bound = (2 * (d + 8) * E * score + (k_len + 64) * E + 2.0 ** -16) * absum + U * np.abs(ref)
    far = np.abs(y - ref) - bound
    assert far.max() <= 0, "worst by %.3g of %.3g" % (far.max(), absum.max())


def _time(sg, ins, outs, n=5):
    import torch
    best = float("inf")
    for _ in range(n):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        sg.run(ins, outs)
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("q_len, heads, d, dtype", [(1024, 8, 64, "bf16"), (1024, 4, 128, "bf16"), (1024, 32, 64, "f32"),
                                                    (8, 1, 64, "bf16"), (8, 1, 128, "f32")])
def test_attention_nan_costs_no_time(q_len, heads, d, dtype):
    """An infinite or NaN value that the rows see, or that a causal mask hides from a few of them, leaves a prompt at
    its speed (ten times at most: the rows that share its tile are formed key by key, over that tile alone)."""
    import torch
    announce("attention of NaN q %d heads %d d %d %s" % (q_len, heads, d, dtype))
    n = 1024
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v = (torch.randn(m, heads * d, generator=g, device=DEV).to(kind) for m in (q_len, n, n))
    host = {"q": np.zeros(q.shape, np.float32), "k": np.zeros(k.shape, np.float32), "v": np.zeros(v.shape, np.float32)}
    _, sg = _engine("attention", host, ["q", "k", "v"], {"batch": 1, "heads": heads, "head_dim": d, "causal": True}, dtype)
    with sg:
        out, clean_out = torch.empty_like(q), torch.empty_like(q)
        _time(sg, [q, k, v], [out])
        clean = _time(sg, [q, k, v], [clean_out])
        for at, value in ((0, float("nan")), (n - q_len, float("inf")), (n - 4, float("nan")), (n - 2, float("-inf"))):
            bad = v.clone()
            bad[at, 1] = value
            t = _time(sg, [q, k, bad], [out])
            assert t <= 10 * clean, "value %g at key %d: %.3f ms, %.3f without" % (value, at, t, clean)
            # the rows before it, and the other columns, are what they were
            seen = torch.arange(q_len, device=DEV) + n - q_len >= at
            assert not torch.isfinite(out[seen, 1]).any()
            keep = torch.ones_like(out, dtype=torch.bool)
            keep[seen, 1] = False
            assert torch.isfinite(out[keep]).all()
            # (their weights may be rounded on one way and not on the other)
            assert ((out[keep] - clean_out[keep]).float().abs() <= 2.0 ** -6 * (1 + clean_out[keep].float().abs())).all()


# ---- plans -----------------------------------------------------------------------

def test_decoder_layer_two_streams(monkeypatch):
    """Launches that do not depend on the one before them on the engine's second stream: the bits of one stream, also
    replayed from a graph."""
    import torch
    from paper_2105_03215_amd import capi, runtime
    wl = _layer(batch=2, tokens=40, encoder_tokens=300)
    monkeypatch.delenv("BYOC_STREAMS", raising=False)
    one = capi.Subgraph(wl.graph, wl.consts, device=0)
    monkeypatch.setenv("BYOC_STREAMS", "2")
    two = capi.Subgraph(wl.graph, wl.consts, device=0)
    monkeypatch.delenv("BYOC_STREAMS")
    s = torch.cuda.Stream(device=DEV)
    with one, two:
        ins, ref = runtime.inputs_for(one, wl.inputs, DEV), runtime.outputs_for(one, DEV)
        torch.cuda.synchronize()
        one.run(ins, ref, s)
        s.synchronize()
        for replay in (False, True, True, True):
            two.set_options(graph_replay=replay)
            out = runtime.outputs_for(two, DEV)
            out[0].fill_(float("nan"))
            torch.cuda.synchronize()
            for _ in range(2):
                two.run(ins, out, s)
            s.synchronize()
            assert torch.equal(ref[0].view(torch.int16), out[0].view(torch.int16))
            torch.mm(torch.ones(64, 64, device=DEV), torch.ones(64, 64, device=DEV))
            torch.cuda.synchronize()
