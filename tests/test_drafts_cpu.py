"""Refusals and host planning of the drafted tokens' composites (no GPU)."""

import json
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

import test_sanitize_cpu as S
from paper_2105_03215_amd import capi, workloads
from paper_2105_03215_amd.capi import ByocError, validate
from test_transformer_bounds_cpu import _mutants
from test_transformer_cpu import _expect, _graph


def _mx(composite="mxdense_bias", x=(3, 40), w=(24, 40), dtype="bf16", **attrs):
    consts = [("w", np.zeros(w, np.float32))] + ([("b", np.zeros(24, np.float32))] if "_bias" in composite else [])
    shapes = {"x": (x, dtype)}
    args = ["x"] + [n for n, _ in consts]
    if "_add" in composite:
        shapes["r"] = ((x[0], w[0]), dtype)
        args.append("r")
    return _graph(composite, shapes, args, attrs, dtype, consts)


def test_mxdense_accepts():
    for name in ("mxdense", "mxdense_bias", "mxdense_bias_add_gelu", "mxdense_add_relu6", "mxdense_leaky"):
        for dtype in ("bf16", "f32"):
            validate(*_mx(name, dtype=dtype))
    validate(*_mx(x=(1, 131072), w=(24, 131072)))


@pytest.mark.parametrize("gc, status, text", [
    (lambda: _mx(w=(24, 48)), "SHAPE", "does not match data"),
    (lambda: _mx("mxdense_add_bias"), "UNSUPPORTED", "unknown composite"),
    (lambda: _mx("mxdense_tanh"), "UNSUPPORTED", "unknown composite"),
    (lambda: _mx("mxdense", x=(1, 131073), w=(24, 131073)), "UNSUPPORTED", "131072"),
    (lambda: _graph("mxdense", {"x": ((3, 40), "bf16"), "w": ((24, 40), "bf16")}, ["x", "w"], {}), "UNSUPPORTED", "constant"),
    (lambda: _graph("mxdense", {"x": ((1, 3, 5, 8), "bf16")}, ["x", "w"], {}, "bf16", [("w", np.zeros((4, 8), np.float32))]),
     "SHAPE", "2-D"),
    (lambda: _mx("mxdense_leaky", alpha=1.5), "PARSE", "alpha"),
    (lambda: _mx("mxdense", x=(2 ** 24, 1), w=(24, 1)), "UNSUPPORTED", "2^32 4-bit codes"),
])
def test_mxdense_refusals(gc, status, text):
    _expect(gc(), status, text)


def test_no_int8_forms():
    for gc in (_mx("mxdense"), _tree(), _rules("mask")):
        g, c = gc
        g["nodes"][0]["out_dtype"] = "int8"
        _expect((g, c), "UNSUPPORTED", "bf16 and f32")


def _tree(dtype="bf16", q=(6, 32), k=(10, 16), v=(10, 16), dk=(6, 16), dv=(6, 16), n=(2,), p=(6,), args=None, **attrs):
    a = dict({"batch": 2, "heads": 4, "kv_heads": 2, "head_dim": 8}, **attrs)
    shapes = {"q": (q, dtype), "k": (k, dtype), "v": (v, dtype), "dk": (dk, dtype), "dv": (dv, dtype), "n": (n, "i32"),
              "p": (p, "i32")}
    return _graph("attention_tree", shapes, args or list(shapes), {key: x for key, x in a.items() if x is not None}, dtype)


def test_attention_tree_accepts():
    validate(*_tree())
    validate(*_tree("f32", scale=0.1))
    validate(*_tree(q=(6, 64), dv=(6, 24), dk=(6, 32), q_col=32, draft_k_col=16, draft_v_col=8))
    validate(*_tree(q=(512, 32), dk=(512, 16), dv=(512, 16), p=(512,)))


@pytest.mark.parametrize("kw, status, text", [
    (dict(batch=None), "PARSE", "are required"),
    (dict(heads=3), "SHAPE", "not a multiple of attrs.kv_heads"),
    (dict(head_dim=12, heads=2, kv_heads=1), "UNSUPPORTED", "multiple of 8"),
    (dict(k_col=8), "SHAPE", "k_col"),
    (dict(draft_k_col=8), "SHAPE", "draft_k_col"),
    (dict(draft_v_col=4), "UNSUPPORTED", "multiple of 8"),
    (dict(dv=(6, 8)), "SHAPE", "draft_v_col"),
    (dict(dk=(5, 16)), "SHAPE", "differ in rows from the queries"),
    (dict(dv=(12, 16)), "SHAPE", "differ in rows from the queries"),
    (dict(dk=(6, 2, 8, 1)), "SHAPE", "must be 2-D"),
    (dict(n=(3,)), "SHAPE", "lengths shape"),
    (dict(p=(5,)), "SHAPE", "parents shape"),
    (dict(causal=True), "UNSUPPORTED", "causal"),
    (dict(dtype="f32", dk=(6, 18)), "UNSUPPORTED", "multiple of 4"),
    (dict(q=(514, 32), dk=(514, 16), dv=(514, 16), p=(514,)), "UNSUPPORTED", "more than 256"),
    (dict(args=["q", "k", "v", "dk", "dv", "n"]), "PARSE", "expects 7"),
    (dict(args=["q", "k", "v", "dk", "dv", "n", "q"]), "SHAPE", "must be an i32"),
    (dict(args=["q", "k", "v", "dk", "p", "n", "p"]), "SHAPE", "must not be i32"),
])
def test_attention_tree_refusals(kw, status, text):
    _expect(_tree(**kw), status, text)


def _rules(rules="penalties_drafts_bias_mask", dtype="bf16", x=(6, 70), batch=2, args=None, strengths_dtype="f32", **shape):
    """shape: an input's other shape."""
    shapes = {"x": (x, dtype)}
    if "penalties" in rules:
        shapes.update(h=((10,), "i32"), pl=((2,), "i32"), n=((2,), "i32"), s=((2, 3), strengths_dtype))
    if "drafts" in rules:
        shapes.update(t=((6,), "i32"), p=((6,), "i32"))
    if "bias" in rules:
        shapes.update(bt=((8,), "i32"), bv=((2, 4), "f32"))
    if "mask" in rules:
        shapes.update(m=((18,), "i32"))
    shapes.update({k: (v, shapes[k][1]) for k, v in shape.items()})
    return _graph("logits_" + rules, shapes, args or list(shapes), {} if batch is None else {"batch": batch}, dtype)


def test_logits_accepts():
    for rules in ("penalties", "penalties_drafts", "bias", "mask", "penalties_bias", "penalties_mask", "bias_mask",
                  "penalties_drafts_bias_mask"):
        for dtype in ("bf16", "f32"):
            validate(*_rules(rules, dtype))
    validate(*_rules("penalties", h=(2 ** 30 - 1024,)))
    validate(*_rules("penalties_bias", h=(2 ** 22 - 1024,), bt=(1022,), bv=(2, 511)))


@pytest.mark.parametrize("kw, status, text", [
    (dict(rules="drafts"), "UNSUPPORTED", "unknown composite"),
    (dict(rules="mask_bias"), "UNSUPPORTED", "unknown composite"),
    (dict(rules=""), "UNSUPPORTED", "unknown composite"),
    (dict(batch=None), "PARSE", "attrs.batch is required"),
    (dict(batch=0), "PARSE", "attrs.batch"),
    (dict(batch=4), "SHAPE", "multiple of attrs.batch"),
    (dict(batch=3), "SHAPE", "history"),
    (dict(h=(11,)), "SHAPE", "history"),
    (dict(pl=(3,)), "SHAPE", "prompt lengths shape"),
    (dict(n=(1,)), "SHAPE", "lengths shape"),
    (dict(s=(2, 2)), "SHAPE", "strengths shape"),
    (dict(strengths_dtype="bf16"), "SHAPE", "must be an f32 input"),
    (dict(t=(5,)), "SHAPE", "drafted tokens shape"),
    (dict(p=(7,)), "SHAPE", "parents shape"),
    (dict(bt=(9,)), "SHAPE", "bias tokens"),
    (dict(bv=(2, 3)), "SHAPE", "bias values shape"),
    (dict(m=(17,)), "SHAPE", "mask shape"),
    (dict(x=(1, 2, 3, 4)), "SHAPE", "2-D"),
    (dict(x=(514, 70), t=(514,), p=(514,), m=(514 * 3,)), "UNSUPPORTED", "more than 256"),
    (dict(rules="mask", args=["x"]), "PARSE", "expects 2"),
    # a table word: 30 bits to count 2^29 tokens, two marks and one bit for the entries; 22, two and 9
    (dict(rules="penalties", h=(2 ** 30,)), "UNSUPPORTED", "536870912 tokens with 0"),
    (dict(rules="penalties_bias", h=(2 ** 22,), bt=(1022,), bv=(2, 511)), "UNSUPPORTED", "2097152 tokens with 511"),
    (dict(rules="bias", x=(1, 2 ** 30 + 1), batch=1, bt=(4,), bv=(1, 4)), "UNSUPPORTED", "2^30 columns"),
    (dict(rules="mask", args=["x", "x"]), "SHAPE", "must be an i32"),
])
def test_logits_refusals(kw, status, text):
    _expect(_rules(**kw), status, text)


def test_parameters_are_read_in_one_way():
    """An f32 input of strengths or biases is no activation, and no output."""
    g, c = _rules("bias", x=(2, 4), batch=2)
    twice = dict(g, nodes=g["nodes"] + [{"name": "z", "composite": "add", "inputs": ["x", "bv"], "attrs": {}, "out_dtype": "bf16"}])
    _expect((twice, c), "UNSUPPORTED", "read as strengths or biases")
    _expect((dict(g, outputs=[{"name": "bv"}]), c), "UNSUPPORTED", "cannot be a subgraph output")
    nodes = [{"name": "z", "composite": "add_relu", "inputs": ["x", "x"], "attrs": {}, "out_dtype": "bf16"}]
    inner = dict(g, nodes=nodes + [dict(g["nodes"][0], inputs=["x", "bt", "z"])])
    _expect((inner, c), "SHAPE", "must be an f32 input of the graph")
    # (a value that one node takes as strengths and another as biases is one input)
    g, c = _rules("penalties_bias", bt=(6,), bv=(2, 3))
    g["nodes"][0]["inputs"][-1] = "s"
    validate(g, c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parameters_are_no_activation_of_their_own_node(dtype):
    """The logits themselves as strengths or bias values of the same node."""
    g, c = _rules("penalties", dtype, x=(2, 3), args=["x", "h", "pl", "n", "x"])
    _expect((g, c), "UNSUPPORTED" if dtype == "f32" else "SHAPE",
            "read as strengths or biases" if dtype == "f32" else "must be an f32 input")
    # (an f32 input of a bf16 graph, which the engine rounds where it is an activation)
    for rules, args, x in (("penalties", ["x", "h", "pl", "n", "x"], (2, 3)), ("bias", ["x", "bt", "x"], (2, 4)),
                           ("penalties_bias", ["x", "h", "pl", "n", "x", "bt", "x"], (2, 3))):
        g, c = _rules(rules, dtype, x=x, args=args, **({"bt": (6,)} if rules == "penalties_bias" else {}))
        g["inputs"][0]["dtype"] = "f32"
        _expect((g, c), "UNSUPPORTED", "read as strengths or biases")


def _steps():
    return [("step", dict(batch=2, drafts=3, cached=5, hidden=64, heads=4, kv_heads=2, ffn=96, vocab=77, history=9)),
            ("step_one", dict(batch=1, drafts=1, cached=1, hidden=64, heads=4, kv_heads=2, ffn=96, vocab=33, history=1)),
            ("step_f32", dict(batch=2, drafts=40, cached=300, hidden=64, heads=4, kv_heads=2, ffn=96, vocab=77, dtype="f32"))]


def test_verify_step_plans():
    """The step validates, and its plan is made before a device is looked for."""
    for _, kw in _steps():
        wl = workloads.build("verify_step", **kw)
        validate(wl.graph, wl.consts)
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(ByocError) as ei:
        capi.Subgraph(wl.graph, wl.consts)
    assert ei.value.status_name == "DEVICE" and "no HIP device" in str(ei.value)


@pytest.mark.slow
@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="host-only sanitizer run (a GPU is visible)")
@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_verify_steps_under_asan_ubsan(tmp_path):
    """The host side under the sanitizers: steps of several shapes, whole and malformed."""
    exe, _ = S._build_driver()
    cases = []
    for name, kw in _steps() + [("step_whole", {})]:
        wl = workloads.build("verify_step", **kw)
        cases.append((name, json.dumps(wl.graph), S._const_lines(wl), True))
    wl = workloads.build("verify_step", **_steps()[0][1])
    for k, text in enumerate(_mutants(wl.graph, random.Random(78), 400)):
        cases.append(("step_mut%d" % k, text, S._const_lines(wl), False))
    for name, text, lines, _ in cases:
        (tmp_path / (name + ".json")).write_text(text)
        (tmp_path / (name + ".consts")).write_text(lines)
    (tmp_path / "list.txt").write_text("".join("%s %s\n" % (tmp_path / (n + ".json"), tmp_path / (n + ".consts"))
                                               for n, _, _, _ in cases))
    (tmp_path / "lsan.supp").write_text("leak:libamdhip64\nleak:libhsa-runtime64\nleak:librocprofiler\nleak:libdrm\n")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1:abort_on_error=0:verify_asan_link_order=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", LSAN_OPTIONS="suppressions=%s" % (tmp_path / "lsan.supp"))
    r = subprocess.run([exe, str(tmp_path / "list.txt")], capture_output=True, text=True, env=env, timeout=900)
    report = r.stdout[-4000:] + r.stderr[-8000:]
    assert r.returncode == 0 and "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, report
    lines = [ln for ln in r.stdout.splitlines() if " validate=" in ln]
    assert len(lines) == len(cases)
    refused = 0
    for (name, _, _, ok), ln in zip(cases, lines):
        v, c = int(ln.split("validate=")[1].split()[0]), int(ln.split("create=")[1].split()[0])
        assert c != S.ST_INTERNAL, ln
        assert c == (S.ST_DEVICE if v == S.ST_OK else v), ln
        assert v == S.ST_OK or not ok, ln
        refused += v != S.ST_OK
    assert refused > 200
