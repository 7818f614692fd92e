"""The drafted tokens' composites where a bound is narrow or a path is seldom taken; rounding bounds as in
test_gpu_drafts."""

import numpy as np
import pytest

import oracle
from oracle import drafts as D
from parity_util import announce
from test_gpu_drafts import DEV, E, U, _check_tree, _close, _engine, _mx_case, _normal, _run, _tree_case

pytestmark = pytest.mark.gpu


# ---- mxdense -------------------------------------------------------------------

TILES = ["256x256_s4", "256x128_s3", "128x128_s4", "128x128_s2", "128x64_s3", "64x64_s4", "32x32_s8"]


def _check_mxdense(m, k, n, dtype, suffix, tile):
    """The product against its definition, on the tile that its launch names."""
    from paper_2105_03215_amd import runtime
    announce("mxdense%s %dx%dx%d %s on %s" % (suffix, m, k, n, dtype, tile))
    r, x, w = _mx_case(m, k, n, dtype, suffix)
    ins, args, consts, rest = {"x": (x, dtype)}, ["x", "w"], [("w", w)], []
    b, res = r.normal(size=n).astype(np.float32), _normal(r, m, n)
    _, mag = D.mxdense(x, w, magnitudes=True)
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
    with _engine("mxdense" + suffix, ins, args, {}, dtype, consts) as sg:
        assert [l["name"] for l in sg.launches()] == ["mx_rows", "mxdense_" + tile]
        arrays = [a for a, _ in ins.values()]
        got, again = runtime.run_once(sg, arrays, DEV)[0], runtime.run_once(sg, arrays, DEV)[0]
    assert np.array_equal(got, again, equal_nan=True)
    ref = oracle.run_node({"composite": "mxdense" + suffix, "attrs": {}, "out_dtype": dtype}, [x, w] + rest, mode="exact")
    _close(got, ref, ((k + 8) * 2 * E + (2.0 ** -18 if "gelu" in suffix else 0)) * mag + 1e-37, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tile", range(7))
@pytest.mark.parametrize("m, k, n, suffix", [
    (70, 40, 40, "_bias"),          # one stage of two steps, two of one
    (270, 250, 330, "_bias_add"),
    (600, 129, 1100, "_gelu"),
    (520, 256, 512, "_add_relu"),   # whole tiles along the channels
    (300, 400, 520, "_bias"),       # rings that the reduction fills, or does not by one stage
    (300, 768, 264, ""),
    (300, 900, 264, "_add"),
])
def test_mxdense_short_reductions_on_every_tile(m, k, n, suffix, tile, dtype, monkeypatch):
    """Reductions shorter than the ring, whose last stages are filled with the last one again, and those about as long."""
    monkeypatch.setenv("BYOC_MXDENSE_TILE", str(tile))
    _check_mxdense(m, k, n, dtype, suffix, TILES[tile])


@pytest.mark.parametrize("tile, m, k, n, suffix", [
    (0, 4400, 512, 4400, "_add"), (1, 2600, 768, 4400, "_bias"), (2, 2100, 1024, 2100, ""), (3, 3000, 512, 3000, "_bias_relu"),
    (4, 3000, 768, 1700, "_add"), (5, 1500, 1024, 1500, "_bias_gelu"), (6, 800, 2048, 800, "_bias"),
])
def test_mxdense_whole_rings_of_several_tiles(tile, m, k, n, suffix, monkeypatch):
    """Reductions of as many stages as the ring has, in workgroups that take several tiles: every fill is the next tile's."""
    monkeypatch.setenv("BYOC_MXDENSE_TILE", str(tile))
    _check_mxdense(m, k, n, "bf16", suffix, TILES[tile])


def test_mxdense_short_reductions_choose_large_tiles():
    """What the ring's shortest form is for: many rows and channels, few columns."""
    _check_mxdense(4096, 128, 4096, "bf16", "_bias_add", TILES[0])


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


@pytest.mark.parametrize("batch, t, lk, h, kv, d, lengths, kind", [
    (1, 256, 40, 1, 1, 256, [33], "chain"),
    (2, 200, 70, 2, 1, 160, [70, 0], "random"),
    (1, 129, 3, 1, 1, 200, [3], "chain"),
    (1, 256, 9, 2, 2, 136, [9], "star"),
])
def test_attention_tree_more_tokens_than_threads(batch, t, lk, h, kv, d, lengths, kind):
    """Paths formed by fewer threads than there are tokens, in several passes a round."""
    announce("attention_tree f32 b %d t %d k %d heads %d/%d d %d %s" % (batch, t, lk, h, kv, d, kind))
    a, attrs = _tree_case(batch, t, lk, h, kv, d, lengths, kind)
    ins = {n: (v, "i32" if v.dtype == np.int32 else "f32") for n, v in a.items()}
    with _engine("attention_tree", ins, list(ins), attrs, "f32") as sg:
        assert sg.launches()[0]["name"] == "attention_tree_rows_f32"  # (128 threads for heads of more than 128 columns)
    _check_tree(a, attrs, "f32")
