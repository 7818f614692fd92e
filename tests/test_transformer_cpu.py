"""Refusals and host planning of the transformer-layer composites (no GPU)."""

import copy
import json

import numpy as np
import pytest

from paper_2105_03215_amd import capi, workloads
from paper_2105_03215_amd.capi import ByocError, validate


def _graph(composite, shapes, args, attrs, dtype="bf16", consts=()):
    """shapes: input name -> (shape, dtype)."""
    return ({"format": "byoc-subgraph", "version": 1,
             "inputs": [{"name": n, "shape": list(s), "dtype": d} for n, (s, d) in shapes.items()],
             "constants": [{"name": n, "index": i, "shape": list(a.shape), "dtype": "f32"}
                           for i, (n, a) in enumerate(consts)],
             "nodes": [{"name": "y", "composite": composite, "inputs": list(args), "attrs": attrs, "out_dtype": dtype}],
             "outputs": [{"name": "y"}]}, [a for _, a in consts])


def _expect(gc, status, fragment):
    with pytest.raises(ByocError) as ei:
        validate(*gc)
    assert ei.value.status_name == status, str(ei.value)
    assert fragment in str(ei.value), str(ei.value)


def _attn(composite="attention_lengths", dtype="bf16", q=(6, 32), k=(10, 16), v=(10, 16), n=(2,), **attrs):
    a = dict({"batch": 2, "heads": 4, "kv_heads": 2, "head_dim": 8}, **attrs)
    shapes = {"q": (q, dtype), "k": (k, dtype), "v": (v, dtype), "n": (n, "i32")}
    args = ["q", "k", "v"] + (["n"] if composite == "attention_lengths" else [])
    return _graph(composite, shapes, args, {key: x for key, x in a.items() if x is not None}, dtype)


def test_attention_accepts():
    validate(*_attn())
    validate(*_attn("attention", "f32"))
    validate(*_attn(kv_heads=1, causal=True, scale=0.5, q_col=0, k_col=8, v_col=8))


@pytest.mark.parametrize("kw, status, text", [
    (dict(batch=None), "PARSE", "are required"),
    (dict(heads=None), "PARSE", "are required"),
    (dict(head_dim=None), "PARSE", "are required"),
    (dict(head_dim=12, heads=2, kv_heads=1), "UNSUPPORTED", "multiple of 8"),
    (dict(head_dim=264), "PARSE", "head_dim"),
    (dict(heads=3), "SHAPE", "not a multiple of attrs.kv_heads"),
    (dict(heads=8), "SHAPE", "q_col"),
    (dict(k_col=8), "SHAPE", "k_col"),
    (dict(v_col=4), "UNSUPPORTED", "multiple of 8"),
    (dict(v_col=-8), "PARSE", "v_col"),
    (dict(batch=4, n=(4,)), "SHAPE", "multiple of attrs.batch"),
    (dict(v=(12, 16)), "SHAPE", "differ in rows"),
    (dict(n=(3,)), "SHAPE", "lengths shape"),
    (dict(scale=0.0), "PARSE", "scale"),
    (dict(scale=1e300), "UNSUPPORTED", "scale"),
    (dict(causal=1), "PARSE", "causal"),
    (dict(dtype="f32", q=(6, 33)), "UNSUPPORTED", "multiple of 4"),
    (dict(q=(6, 32, 1, 1)), "SHAPE", "2-D"),
])
def test_attention_refusals(kw, status, text):
    _expect(_attn(**kw), status, text)


def test_attention_argument_kinds():
    g, c = _attn()
    for args, text in ((["q", "k", "v"], "expects 4"), (["q", "k", "v", "q"], "must be an i32 input"),
                       (["n", "k", "v", "n"], "must not be i32")):
        g2 = copy.deepcopy(g)
        g2["nodes"][0]["inputs"] = args
        _expect((g2, c), "SHAPE" if "i32" in text else "PARSE", text)
    g2 = copy.deepcopy(g)
    g2["outputs"] = [{"name": "n"}]
    _expect((g2, c), "UNSUPPORTED", "i32 input cannot be")
    g2 = copy.deepcopy(g)
    g2["inputs"][3]["shape"] = [2, 1]
    _expect((g2, c), "UNSUPPORTED", "rank must be 1 for i32")
    g2 = copy.deepcopy(g)
    g2["inputs"][0]["dtype"] = "i32"
    _expect((g2, c), "UNSUPPORTED", "rank must be 1 for i32")
    g2 = copy.deepcopy(g)
    g2["inputs"][3]["dtype"] = "f32"
    _expect((g2, c), "UNSUPPORTED", "rank must be 2 or 4")


def _rot(composite="rotary", dtype="bf16", x=(5, 48), p=(5,), weights=(), args=None, **attrs):
    a = dict({"heads": 2, "kv_heads": 1, "head_dim": 16}, **attrs)
    consts = [("w%d" % i, np.ones(n, np.float32)) for i, n in enumerate(weights)]
    names = args or ["x"] + [n for n, _ in consts] + ["p"]
    return _graph(composite, {"x": (x, dtype), "p": (p, "i32")}, names,
                  {key: v for key, v in a.items() if v is not None}, dtype, consts)


def test_rotary_accepts():
    validate(*_rot())
    validate(*_rot(dtype="f32", x=(5, 51), layout="interleaved", rotary_dim=6, base=500000.0))
    validate(*_rot("qk_norm_rotary", weights=(16, 16)))
    validate(*_rot("qk_norm_rotary", weights=(16,), kv_heads=0))
    for sc in ({"type": "linear", "factor": 2}, {"type": "ntk", "factor": 2.5},
               {"type": "yarn", "factor": 8, "original_length": 4096, "beta_fast": 16, "beta_slow": 2,
                "attention_factor": 1.5}):
        validate(*_rot(scaling=sc))


@pytest.mark.parametrize("kw, status, text", [
    (dict(heads=None), "PARSE", "are required"),
    (dict(head_dim=15), "UNSUPPORTED", "even"),
    (dict(head_dim=514), "PARSE", "head_dim"),
    (dict(rotary_dim=18), "PARSE", "rotary_dim"),
    (dict(rotary_dim=5), "UNSUPPORTED", "even"),
    (dict(kv_heads=2), "SHAPE", "do not fit"),
    (dict(layout="pairs"), "PARSE", "layout"),
    (dict(layout=3), "PARSE", "layout"),
    (dict(base=1.0), "PARSE", "above 1"),
    (dict(base=-2.0), "PARSE", "base"),
    (dict(p=(4,)), "SHAPE", "positions shape"),
    (dict(eps=0), "PARSE", "eps"),
    (dict(scaling="linear"), "PARSE", "scaling"),
    (dict(scaling={"type": "linear"}), "PARSE", "factor missing"),
    (dict(scaling={"type": "linear", "factor": 0.5}), "PARSE", "at least 1"),
    (dict(scaling={"type": "other", "factor": 2}), "UNSUPPORTED", "scaling.type"),
    (dict(scaling={"type": "yarn", "factor": 2}), "PARSE", "original_length"),
    (dict(scaling={"type": "yarn", "factor": 2, "original_length": 64, "beta_fast": 1.0}), "PARSE", "beta_fast"),
    (dict(scaling={"type": "ntk", "factor": 1e308}), "PARSE", "too large"),
    (dict(composite="qk_norm_rotary", weights=(16,)), "PARSE", "weight"),
    (dict(composite="qk_norm_rotary", weights=(16, 8)), "SHAPE", "norm weight"),
    (dict(composite="qk_norm_rotary", weights=()), "PARSE", "expects"),
    (dict(args=["x", "x"]), "SHAPE", "must be an i32 input"),
    (dict(args=["p", "p"]), "SHAPE", "must not be i32"),
    (dict(args=["x"]), "PARSE", "expects 2"),
])
def test_rotary_refusals(kw, status, text):
    _expect(_rot(**kw), status, text)


def _qd(composite="qdense_bias", x=(5, 24), w=(7, 24), b=(7,), dtype="bf16", **extra):
    consts = [("w", np.ones(w, np.float32))] + ([("b", np.ones(b, np.float32))] if "bias" in composite else [])
    shapes = {"x": (x, dtype)}
    shapes.update(extra)
    return _graph(composite, shapes, ["x", "w"] + (["b"] if "bias" in composite else []) + list(extra), {}, dtype, consts)


def test_qdense_accepts_and_refuses():
    validate(*_qd())
    validate(*_qd("qdense", dtype="f32"))
    validate(*_qd("qdense_bias_add_gelu", r=((5, 7), "bf16")))
    validate(*_qd("qdense_leaky"))
    _expect(_qd(w=(7, 23)), "SHAPE", "does not match data")
    _expect(_qd(b=(8,)), "SHAPE", "bias shape")
    _expect(_qd("qdense_add", r=((5, 8), "bf16")), "SHAPE", "residual shape")
    _expect(_qd(x=(5, 24, 1, 1)), "SHAPE", "2-D")
    _expect(_qd("qdense_swish"), "UNSUPPORTED", "unknown composite")
    _expect(_qd("qdense", x=(1, 131080), w=(1, 131080)), "UNSUPPORTED", "131072")


@pytest.mark.parametrize("gc", [_qd(dtype="bf16"), _rot(), _attn()])
def test_not_in_int8_graphs(gc):
    g = copy.deepcopy(gc[0])
    g["nodes"][0]["out_dtype"] = "int8"
    _expect((g, gc[1]), "UNSUPPORTED", "only in bf16 and f32 graphs")


def test_quant_parameters_refused_on_index_inputs():
    g, c = _rot()
    g["inputs"][1]["quant"] = {"scale": 1.0, "zero_point": 0}
    _expect((g, c), "UNSUPPORTED", "i32")


def test_decoder_layer_plans():
    """The whole layer validates, and its plan is made before a device is looked for."""
    wl = workloads.build("decoder_layer", batch=2, tokens=3, encoder_tokens=5, hidden=64, heads=4, kv_heads=2, ffn=96)
    validate(wl.graph, wl.consts)
    validate(json.dumps(wl.graph), wl.consts)
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(ByocError) as ei:
        capi.Subgraph(wl.graph, wl.consts)
    assert ei.value.status_name == "DEVICE" and "no HIP device" in str(ei.value)
