"""What the transformer-layer composites refuse and plan at the edges of their ranges (no GPU)."""

import copy
import json
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

import test_sanitize_cpu as S
from paper_2105_03215_amd import workloads
from paper_2105_03215_amd.capi import ByocError, validate
from test_oracle_quant import _tiny_int8_graph


def test_index_inputs_are_refused_in_int8_graphs():
    """No int8 composite reads one, and the int8 planner lays every input out as activations."""
    g, consts = _tiny_int8_graph()
    validate(g, consts)
    for at in (0, len(g["inputs"])):
        bad = dict(g, inputs=list(g["inputs"]))
        bad["inputs"].insert(at, {"name": "positions", "shape": [4], "dtype": "i32"})
        with pytest.raises(ByocError) as ei:
            validate(bad, consts)
        assert ei.value.status_name == "UNSUPPORTED"
        assert "input positions: i32 inputs only in bf16 and f32 graphs" in str(ei.value)


def test_index_inputs_that_nothing_reads_are_accepted_elsewhere():
    for dtype in ("bf16", "f32"):
        w = np.ones((8, 16), np.float32)
        validate({"format": "byoc-subgraph", "version": 1,
                  "inputs": [{"name": "p", "shape": [4], "dtype": "i32"}, {"name": "x", "shape": [2, 16], "dtype": dtype}],
                  "constants": [{"name": "w", "index": 0, "shape": [8, 16], "dtype": "f32"}],
                  "nodes": [{"name": "y", "composite": "dense", "inputs": ["x", "w"], "attrs": {}, "out_dtype": dtype}],
                  "outputs": [{"name": "y"}]}, [w])


def _mutants(base, rng, count):
    """Layers with an attribute, a type or a shape that does not belong there."""
    values = [0, -1, 1, 3, 7, 8, 24, 255, 256, 257, 513, 2 ** 20, 2 ** 31, 2 ** 63, 1.5, 1e-300, 1e300, "x", None, True, [], [8], {},
              {"type": "yarn"}, {"type": "yarn", "factor": 2, "original_length": 8}, {"type": "ntk", "factor": 1e300},
              {"type": "linear", "factor": -1}]
    attrs = ["batch", "heads", "kv_heads", "head_dim", "rotary_dim", "q_col", "k_col", "v_col", "scale", "causal", "layout",
             "base", "scaling", "eps"]
    out = []
    for i in range(count):
        g = copy.deepcopy(base)
        node = rng.choice(g["nodes"])
        kind = i % 5
        if kind == 0:
            node = rng.choice([n for n in g["nodes"] if n.get("attrs")])
            node["attrs"][rng.choice(attrs)] = rng.choice(values)
        elif kind == 1:
            node["composite"] = rng.choice(["qdense", "qdense_bias_add_gelu", "rotary", "qk_norm_rotary", "attention",
                                            "attention_lengths", "dense_bias", "add"])
        elif kind == 2:
            names = [d["name"] for d in g["inputs"] + g["constants"]] + [n["name"] for n in g["nodes"]]
            node["inputs"][rng.randrange(len(node["inputs"]))] = rng.choice(names)
        elif kind == 3:
            d = rng.choice(g["inputs"])
            d["shape"] = rng.choice([[], [0], [1], [2 ** 31], [2, 3], [6, 1], [2 ** 20, 2 ** 20], [1, 2, 3, 4]])
        else:
            rng.choice(g["inputs"])["dtype"] = rng.choice(["i32", "int32", "f32", "bf16", "i8", 3, None])
        if rng.random() < 0.3:
            rng.choice(g["nodes"])["out_dtype"] = rng.choice(["f32", "int8", "bf16"])
        out.append(json.dumps(g))
    return out


@pytest.mark.slow
@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="host-only sanitizer run (a GPU is visible)")
@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_decoder_layers_under_asan_ubsan(tmp_path):
    """The host side under the sanitizers, on decoder layers, on index inputs beside int8 nodes and on malformed ones."""
    exe, _ = S._build_driver()
    cases = []
    for name, kw in (("layer", dict(batch=2, tokens=3, encoder_tokens=5, hidden=64, heads=4, kv_heads=2, ffn=96)),
                     ("layer_whole", dict()), ("layer_token", dict(tokens=1, start=900))):
        wl = workloads.build("decoder_layer", **kw)
        cases.append((name, json.dumps(wl.graph), S._const_lines(wl), True))
    wl = workloads.build("decoder_layer", batch=2, tokens=3, encoder_tokens=5, hidden=64, heads=4, kv_heads=2, ffn=96)
    for k, text in enumerate(_mutants(wl.graph, random.Random(77), 400)):
        cases.append(("layer_mut%d" % k, text, S._const_lines(wl), False))
    g, consts = _tiny_int8_graph()
    lines = "\n".join(" ".join(["0", str(a.ndim)] + [str(n) for n in a.shape]) for a in consts) + "\n"
    cases.append(("int8_index", json.dumps(dict(g, inputs=g["inputs"] + [{"name": "positions", "shape": [4], "dtype": "i32"}])),
                  lines, False))
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
    assert refused > 200 and lines[-1].split("validate=")[1].split()[0] == "3", (refused, lines[-1])
