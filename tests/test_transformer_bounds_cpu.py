"""What the transformer-layer composites refuse and plan at the edges of their ranges (no GPU)."""

import numpy as np
import pytest

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
