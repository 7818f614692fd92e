"""The drafted tokens' composites where a bound is narrow or a path is seldom taken; rounding bounds as in
test_gpu_drafts."""

import numpy as np
import pytest

from oracle import drafts as D
from parity_util import announce
from test_gpu_drafts import E, U, _normal, _run, _tree_case

pytestmark = pytest.mark.gpu


# ---- attention of a tree ----------------------------------------------------------

@pytest.mark.parametrize("batch, t, lk, h, kv, d, lengths", [
    (1, 40, 200, 2, 2, 32, [200]),            # tiles of 64 rows
    (1, 40, 200, 2, 2, 64, [177]),
    (41, 33, 70, 8, 8, 24, None),             # tiles of 128 rows
    (41, 33, 70, 8, 8, 64, None),
    (2, 40, 200, 4, 2, 96, [200, 3]),
    (2, 12, 200, 8, 2, 128, [200, 64]),
    (1, 40, 100, 1, 1, 160, [100]),
    (1, 40, 100, 1, 1, 256, [99]),
    (2, 24, 3000, 8, 2, 128, [3000, 700]),    # split key axes
    (1, 24, 1000, 4, 1, 128, [1000]),
    (1, 150, 33, 2, 2, 128, [33]),            # drafted keys of several tiles
    (3, 7, 90, 4, 2, 128, [90, 0, 31]),       # few rows
])
def test_attention_tree_weights_are_not_rounded_to_bf16(batch, t, lk, h, kv, d, lengths):
    """Outputs near zero, of values of either sign, leave the error of the weights alone: 2^-16 of each, two
    roundings to bf16 one after the other, where one alone is 2^-8."""
    announce("attention_tree weights b %d t %d k %d heads %d/%d d %d" % (batch, t, lk, h, kv, d))
    a, attrs = _tree_case(batch, t, lk, h, kv, d, lengths, "random", seed=6)
    # (scores near each other, so that their own rounding stays below that of the weights)
    a["q"] = _normal(np.random.default_rng(d + t), *a["q"].shape, std=0.02)
    ins = {n: (v, "i32" if v.dtype == np.int32 else "bf16") for n, v in a.items()}
    y = _run("attention_tree", ins, list(ins), attrs, "bf16")
    ref, absum, score = D.attention_tree(attrs, *a.values(), magnitudes=True)
    bound = (2 * (d + 8) * E * score + (lk + t + 200) * E + 2.0 ** -16) * absum + U * np.abs(ref)
    far = np.abs(y - ref) - bound
    assert far.max() <= 0, "%d of %d, worst by %.3g of %.3g" % ((far > 0).sum(), far.size, far.max(), absum.max())
