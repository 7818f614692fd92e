"""Cases of the transformer-layer composites: `qdense` (8-bit matrix product with scales for each token and
channel), `rotary` / `qk_norm_rotary` (position rotation of packed heads, with the heads' norms) and
`attention` (cross and causal self attention with lengths), each in a plain torch form and as a user calls it."""

import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ------------------------------------------------------------------

def _q(name, m, k, n, dtype="bf16", bias=True, residual=False, act="none"):
    return {"name": name, "op": "qdense", "dtype": dtype, "m": m, "k": k, "n": n, "bias": bias,
            "residual": residual, "act": act}


def _r(name, m, heads, kv_heads, head_dim, rotary_dim, dtype="bf16", norm=False, layout="half", scaling="none",
       factor=1.0, base=10000.0, top=4096, extra=0):
    return {"name": name, "op": "rotary", "dtype": dtype, "m": m, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rotary_dim": rotary_dim, "norm": norm, "layout": layout, "scaling": scaling,
            "factor": factor, "base": base, "top": top, "extra": extra}


def _a(name, batch, q_len, k_len, heads, kv_heads, head_dim, dtype="bf16", causal=False, lengths="none",
       packed="kv"):
    return {"name": name, "op": "attention", "dtype": dtype, "batch": batch, "q_len": q_len, "k_len": k_len,
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "lengths": lengths,
            "packed": packed}


def listed():
    return [
        # one token through the feed-forward up-projection of a BERT-base layer: latency alone
        _q("qdense_one_token", 1, 768, 3072, act="gelu"),
        # a decoding batch against a wide layer: the weights' bytes
        _q("qdense_decode_batch", 24, 4096, 12288),
        # the repository's BERT feed-forward block, 8 x 128 tokens
        _q("qdense_bert_ffn", 1024, 768, 3072, act="gelu"),
        # an fp32 graph with sizes that fill no tile, with a residual
        _q("qdense_odd_f32", 1531, 1000, 2056, dtype="f32", residual=True),
        # a long prompt through a wide projection: the matrix cores
        _q("qdense_prompt", 8192, 4096, 8192, residual=True),
        # one token of each of four sequences, heads of a BERT-base layer
        _r("rotary_tokens", 4, 12, 12, 64, 64, extra=12),
        # a prompt of 2 x 4096 tokens from the packed q|k|v projection, normed, in a context extended 8 times
        _r("qk_norm_rotary_prompt", 8192, 32, 8, 128, 128, norm=True, scaling="yarn", factor=8.0, top=32768, extra=8),
        # part of the head, neighbouring pairs, fp32, an odd number of tokens
        _r("rotary_part_f32", 2047, 16, 16, 80, 32, dtype="f32", layout="interleaved", scaling="linear", factor=4.0,
           top=16384),
        # one decoder step of a batch over its encoders' states of different lengths
        _a("cross_one_token", 16, 1, 1500, 12, 12, 64, lengths="ragged"),
        # one token over long contexts, four query heads to a key head
        _a("decode_long", 4, 1, 32768, 32, 8, 128, lengths="ragged"),
        # decoder prompts over encoder states of different lengths, sizes that fill no tile
        _a("cross_prompt", 8, 449, 1027, 12, 12, 64, lengths="ragged"),
        # causal self attention of two 4096-token prompts, straight from the rotated q|k and the projection's v
        _a("self_causal", 2, 4096, 4096, 32, 8, 128, causal=True, packed="self"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["qdense", "rotary", "attention", "attention"])
    if op == "qdense":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        unit = rng.choice([8, 8, 8, 1])
        while True:
            m, k, n = _log(rng, 1, 8192), _log(rng, 64, 8192), _log(rng, 64, 12288)
            k, n = max(unit, k // unit * unit), max(unit, n // unit * unit)
            if 2 * m * k * n <= (2 * 8192 * 4096 * 8192 if dtype == "bf16" else 1 << 36):
                break
        c = _q("", m, k, n, dtype, rng.random() < 0.7, rng.random() < 0.3, rng.choice(["none", "gelu", "relu"]))
    elif op == "rotary":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        m, head_dim = _log(rng, 1, 8192), rng.choice([32, 48, 64, 80, 96, 128, 128, 256])
        heads = rng.choice([1, 2, 6, 8, 12, 16, 20, 32])
        kv = rng.choice([0, 1, heads, max(1, heads // 4)])
        while m * (heads + kv) * head_dim > 8192 * 40 * 128:
            m //= 2
        scaling = rng.choice(["none", "linear", "ntk", "yarn"])
        c = _r("", max(1, m), heads, kv, head_dim, head_dim if rng.random() < 0.6 else head_dim // 4 * 2, dtype,
               rng.random() < 0.5, rng.choice(["half", "interleaved"]), scaling,
               1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 2.5]), rng.choice([10000.0, 500000.0]),
               _log(rng, 16, 65536), rng.choice([0, 1, kv]))
    else:
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        head_dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
        heads, kv = rng.choice([(8, 8), (12, 12), (32, 8), (16, 1), (20, 4), (3, 3)])
        causal = rng.random() < 0.4
        while True:
            batch, q_len, k_len = _log(rng, 1, 16), rng.choice([1, 1, _log(rng, 2, 4096)]), _log(rng, 1, 32768)
            if causal and rng.random() < 0.7:
                q_len = k_len = min(k_len, 4096)
            pairs = batch * heads * q_len * k_len
            if (batch * k_len * kv * head_dim <= 4 * 32768 * 8 * 128 and pairs <= 2 * 32 * 4096 * 4096 // 2 and
                    4 * pairs * head_dim <= (140e9 if dtype == "bf16" else 8e9)):
                break
        c = _a("", batch, q_len, k_len, heads, kv, head_dim, dtype, causal, rng.choice(["none", "ragged"]),
               "self" if q_len == k_len else rng.choice(["kv", "apart"]))
    del c["name"]
    return c


# ---- what a program has in hand ------------------------------------------------

def _lengths(c):
    """Valid keys of each sequence: all of them, or spread over the range, with an empty one in larger batches."""
    b, n = c["batch"], c["k_len"]
    if c["lengths"] == "none":
        return [n] * b
    got = [max(1, round(n * ((0.73 + 0.617 * i) % 1.0))) for i in range(b)]
    if b > 1:
        got[0] = n
    if b >= 6:
        got[b - 2] = 0
    return got


def _turned(c, seed):
    got = _lengths(c)
    at = seed % len(got)
    return got[at:] + got[:at]


def _theta(c):
    """Angle per position of each pair, and the factor on the rotated values, in Python's 64-bit floats."""
    rd, base, f = c["rotary_dim"], c["base"], c["factor"]
    if c["scaling"] == "ntk" and rd > 2:
        base = base * f ** (rd / (rd - 2))
    theta = [base ** (-2.0 * i / rd) for i in range(rd // 2)]
    if c["scaling"] == "linear":
        return [t / f for t in theta], 1.0
    if c["scaling"] != "yarn":
        return theta, 1.0

    def dim(rotations):
        return rd * math.log(_ORIGINAL / (rotations * 2 * math.pi)) / (2 * math.log(base))

    low, high = max(math.floor(dim(32.0)), 0), min(math.ceil(dim(1.0)), rd - 1)
    ramp = [min(1.0, max(0.0, (i - low) / max(high - low, 1e-3))) for i in range(rd // 2)]
    return [t * (1 - r) + t / f * r for t, r in zip(theta, ramp)], 0.1 * math.log(f) + 1.0


_ORIGINAL = 4096  # the context that scaled rotations were trained on


def _data(case, seed):
    """The case's tensors, from the seed alone."""
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=_DT[c["dtype"]]):
        return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)

    if c["op"] == "qdense":
        d = {"x": normal(c["m"], c["k"]), "w": normal(c["n"], c["k"], std=0.02, dtype=torch.bfloat16)}
        # a few channels of the activations stand out, as they do in transformers
        d["x"][:, torch.randint(0, c["k"], (max(1, c["k"] // 256),), generator=g, device="cuda")] *= 8
        d["bias"] = normal(c["n"], std=0.02, dtype=torch.float32) if c["bias"] else None
        d["residual"] = normal(c["m"], c["n"]) if c["residual"] else None
        return d
    if c["op"] == "rotary":
        width = (c["heads"] + c["kv_heads"] + c["extra"]) * c["head_dim"]
        d = {"x": normal(c["m"], width),
             "positions": torch.randint(0, c["top"], (c["m"],), generator=g, device="cuda", dtype=torch.int32)}
        d["wq"] = 1 + normal(c["head_dim"], std=0.1, dtype=torch.float32)
        d["wk"] = 1 + normal(c["head_dim"], std=0.1, dtype=torch.float32)
        return d
    b, hd, kd = c["batch"], c["heads"] * c["head_dim"], c["kv_heads"] * c["head_dim"]
    d = {"lengths": torch.tensor(_turned(c, seed), device="cuda", dtype=torch.int32)}
    if c["packed"] == "self":  # rotated q|k, and v where the projection left it
        d["q"] = d["k"] = normal(b * c["q_len"], hd + kd)
        d["v"] = normal(b * c["k_len"], hd + 2 * kd)
        d["cols"] = (0, hd, hd + kd)
    elif c["packed"] == "kv":
        d["q"] = normal(b * c["q_len"], hd)
        d["k"] = d["v"] = normal(b * c["k_len"], 2 * kd)
        d["cols"] = (0, 0, kd)
    else:
        d["q"], d["k"], d["v"] = normal(b * c["q_len"], hd), normal(b * c["k_len"], kd), normal(b * c["k_len"], kd)
        d["cols"] = (0, 0, 0)
    return d


def _codes(t):
    """Symmetric 8-bit codes of each row and its largest magnitude."""
    top = t.abs().amax(dim=1, keepdim=True)
    return torch.round(torch.where(top > 0, 127 * t / top, torch.zeros_like(t))), top


def prepare(case, seed):
    c = case
    s = {"case": c, **_data(c, seed)}
    if own:
        s.update(_engine(c, s))
    elif c["op"] == "qdense":  # the layer's quantised weights
        codes, top = _codes(s["w"].float())
        s["codes"], s["scales"] = codes.to(torch.int8), (top / 127).reshape(1, -1)
    elif c["op"] == "rotary":  # the model's table of rotations
        theta, mag = _theta(c)
        a = torch.arange(c["top"], device="cuda", dtype=torch.float64)[:, None] * torch.tensor(
            theta, device="cuda", dtype=torch.float64)
        s["cos"], s["sin"] = (a.cos() * mag).float(), (a.sin() * mag).float()
    if c["op"] == "qdense":
        del s["w"]
    return s


def _engine(c, s):
    """The serialized composite, its engine and the output buffer."""
    from paper_2105_03215_amd import capi
    dt = c["dtype"]
    consts, entries = [], []

    def const(name, t):
        entries.append({"name": name, "index": len(consts), "shape": list(t.shape),
                        "dtype": "bf16" if t.dtype == torch.bfloat16 else "f32"})
        consts.append(t.cpu())
        return name

    def tensor(name, t, dtype=dt):
        return {"name": name, "shape": list(t.shape), "dtype": dtype}

    if c["op"] == "qdense":
        name = "qdense" + ("_bias" if c["bias"] else "") + ("_add" if c["residual"] else "")
        name += "" if c["act"] == "none" else "_" + c["act"]
        ins, args = [tensor("x", s["x"])], ["x", const("w", s["w"])]
        feed = [s["x"]]
        if c["bias"]:
            args.append(const("b", s["bias"]))
        if c["residual"]:
            ins.append(tensor("r", s["residual"]))
            feed.append(s["residual"])
            args.append("r")
        attrs, shape = {}, [c["m"], c["n"]]
    elif c["op"] == "rotary":
        name = "qk_norm_rotary" if c["norm"] else "rotary"
        ins, feed = [tensor("x", s["x"]), tensor("p", s["positions"], "i32")], [s["x"], s["positions"]]
        args = ["x"]
        if c["norm"]:
            args.append(const("wq", s["wq"]))
            if c["kv_heads"]:
                args.append(const("wk", s["wk"]))
        args.append("p")
        attrs = {"heads": c["heads"], "kv_heads": c["kv_heads"], "head_dim": c["head_dim"],
                 "rotary_dim": c["rotary_dim"], "layout": c["layout"], "base": c["base"]}
        if c["scaling"] != "none":
            attrs["scaling"] = {"type": c["scaling"], "factor": c["factor"]}
            if c["scaling"] == "yarn":
                attrs["scaling"]["original_length"] = _ORIGINAL
        shape = [c["m"], (c["heads"] + c["kv_heads"]) * c["head_dim"]]
    else:
        ragged = c["lengths"] != "none"
        name = "attention_lengths" if ragged else "attention"
        ins, feed, args = [], [], []
        for key in "qkv":
            same = [j for j, t in enumerate(feed) if t is s[key]]
            if not same:
                ins.append(tensor(key, s[key]))
                feed.append(s[key])
            args.append(ins[same[0]]["name"] if same else key)
        if ragged:
            ins.append(tensor("n", s["lengths"], "i32"))
            feed.append(s["lengths"])
            args.append("n")
        attrs = {"batch": c["batch"], "heads": c["heads"], "kv_heads": c["kv_heads"], "head_dim": c["head_dim"],
                 "causal": c["causal"], "q_col": s["cols"][0], "k_col": s["cols"][1], "v_col": s["cols"][2]}
        shape = [c["batch"] * c["q_len"], c["heads"] * c["head_dim"]]
    graph = {"format": "byoc-subgraph", "version": 1, "inputs": ins, "constants": entries,
             "nodes": [{"name": "y", "composite": name, "inputs": args, "attrs": attrs, "out_dtype": dt}],
             "outputs": [{"name": "y", "dtype": dt}]}
    return {"engine": capi.Subgraph(graph, consts, device=torch.cuda.current_device()), "feed": feed,
            "out": [torch.empty(shape, device="cuda", dtype=_DT[dt])]}


# ---- one pass -------------------------------------------------------------------

def run(state):
    if own:
        state["engine"].run(state["feed"], state["out"])
        return state["out"][0]
    return {"qdense": _plain_qdense, "rotary": _plain_rotary, "attention": _plain_attention}[state["case"]["op"]](state)


def _plain_qdense(s):
    c = s["case"]
    codes, top = _codes(s["x"].float())
    y = torch.matmul(codes, s["codes"].float().t()) * (top / 127) * s["scales"]
    if c["bias"]:
        y = y + s["bias"]
    if c["residual"]:
        y = y + s["residual"].float()
    if c["act"] == "relu":
        y = y.clamp_min(0)
    elif c["act"] == "gelu":
        y = 0.5 * y * torch.erfc(y * -math.sqrt(0.5))
    return y.to(_DT[c["dtype"]])


def _plain_rotary(s):
    c = s["case"]
    h, kv, d, rd = c["heads"], c["kv_heads"], c["head_dim"], c["rotary_dim"]
    x = s["x"][:, :(h + kv) * d].float().view(-1, h + kv, d)
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(dim=2, keepdim=True) + 1e-6)
        x = x * torch.cat([s["wq"].expand(h, d), s["wk"].expand(kv, d)])
    p = s["positions"].long()
    cos, sin = s["cos"][p][:, None, :], s["sin"][p][:, None, :]
    part, rest = x[..., :rd], x[..., rd:]
    if c["layout"] == "half":
        a, b = part[..., :rd // 2], part[..., rd // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=2)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=3).flatten(2)
    return torch.cat([turned, rest], dim=2).reshape(c["m"], -1).to(_DT[c["dtype"]])


def _heads(t, c, n, col, heads):
    return t.view(c["batch"], n, -1)[..., col:col + heads * c["head_dim"]].reshape(c["batch"], n, heads, c["head_dim"])


def _allowed(c, lengths):
    """[batch, q_len, k_len]: which keys each query may see."""
    j = torch.arange(c["k_len"], device=lengths.device)
    n = lengths.long()[:, None, None]
    if c["causal"]:
        i = torch.arange(c["q_len"], device=lengths.device)[:, None]
        n = torch.minimum(n, n - c["q_len"] + i + 1)
    return (j < n).expand(c["batch"], c["q_len"], c["k_len"])


def _plain_attention(s):
    c = s["case"]
    b, lq, lk, h, kv, d = (c[k] for k in ("batch", "q_len", "k_len", "heads", "kv_heads", "head_dim"))
    q = _heads(s["q"], c, lq, s["cols"][0], h).float().permute(0, 2, 1, 3).reshape(b, kv, h // kv * lq, d)
    k = _heads(s["k"], c, lk, s["cols"][1], kv).float().permute(0, 2, 3, 1).contiguous()
    v = _heads(s["v"], c, lk, s["cols"][2], kv).float().permute(0, 2, 1, 3).contiguous()
    score = torch.matmul(q * (1 / math.sqrt(d)), k).view(b, h, lq, lk)
    score = score.masked_fill(~_allowed(c, s["lengths"])[:, None], -math.inf)
    score = torch.exp(score - score.amax(dim=3, keepdim=True).clamp_min(-1e30))
    total = score.sum(dim=3, keepdim=True)
    out = torch.matmul(score.view(b, kv, h // kv * lq, lk), v).view(b, h, lq, d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    return out.permute(0, 2, 1, 3).reshape(b * lq, h * d).to(_DT[c["dtype"]])


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "qdense":
        m, k, n = c["m"], c["k"], c["n"]
        return {"bytes": m * k * es + n * k + 4 * n * (2 if c["bias"] else 1) + m * n * es * (2 if c["residual"] else 1),
                "flops": 2 * m * n * k}
    if c["op"] == "rotary":
        e = c["m"] * (c["heads"] + c["kv_heads"]) * c["head_dim"]
        return {"bytes": 2 * e * es + 4 * c["m"], "flops": e * (7 if c["norm"] else 3)}
    lens = _lengths(c)
    lq, d = c["q_len"], c["head_dim"]
    if c["causal"]:  # query i sees n - q_len + i + 1 keys
        pairs = sum((n * (n + 1) - max(0, n - lq) * (max(0, n - lq) + 1)) // 2 for n in lens)
    else:
        pairs = sum(lens) * lq
    return {"bytes": es * d * (2 * c["batch"] * lq * c["heads"] + 2 * sum(lens) * c["kv_heads"]) + 4 * c["batch"],
            "flops": 4 * pairs * c["heads"] * d}


# ---- the definitions, in 64 bits ----------------------------------------------------

def exact(case, seed):
    c = case
    d = _data(c, seed)
    if c["op"] == "qdense":
        x, w = d["x"].double(), d["w"].double()
        ax, aw = x.abs().max(dim=1).values, w.abs().max(dim=1).values
        qx = (127.0 * x / torch.where(ax > 0, ax, torch.ones_like(ax))[:, None]).round()
        qw = (127.0 * w / torch.where(aw > 0, aw, torch.ones_like(aw))[:, None]).round()
        y = (qx @ qw.t()) * torch.outer(ax / 127.0, aw / 127.0)
        if d["bias"] is not None:
            y += d["bias"].double()
        if d["residual"] is not None:
            y += d["residual"].double()
        if c["act"] == "gelu":
            return y * torch.special.ndtr(y)
        return torch.relu(y) if c["act"] == "relu" else y
    if c["op"] == "rotary":
        n, dim, rd = c["heads"] + c["kv_heads"], c["head_dim"], c["rotary_dim"]
        x = d["x"].double()[:, :n * dim].reshape(c["m"], n, dim)
        if c["norm"]:
            x = x / (x.pow(2).sum(2, keepdim=True) / dim + 1e-6).sqrt()
            x[:, :c["heads"]] *= d["wq"].double()
            x[:, c["heads"]:] *= d["wk"].double()
        theta, mag = _theta(c)
        angle = torch.outer(d["positions"].double(), torch.tensor(theta, device="cuda", dtype=torch.float64))
        turn = torch.polar(torch.full_like(angle, mag), angle)[:, None]
        first = torch.arange(0, rd // 2, device="cuda")
        second = first + rd // 2
        if c["layout"] == "interleaved":
            first, second = 2 * first, 2 * first + 1
        z = torch.complex(x[..., first], x[..., second]) * turn
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        return y.reshape(c["m"], n * dim)
    b, lq, lk, h, dim = c["batch"], c["q_len"], c["k_len"], c["heads"], c["head_dim"]
    out = torch.zeros(b, lq, h, dim, device="cuda", dtype=torch.float64)
    for i, n in enumerate(_turned(c, seed)):
        seen = torch.full((lq,), n, device="cuda")
        if c["causal"]:
            seen = n - lq + 1 + torch.arange(lq, device="cuda")
        empty = seen <= 0
        hidden = torch.arange(n, device="cuda")[None] >= seen[:, None]
        for j in range(h if n else 0):
            at = j // (h // c["kv_heads"]) * dim
            q = d["q"][i * lq:(i + 1) * lq, d["cols"][0] + j * dim:][:, :dim].double()
            k = d["k"][i * lk:i * lk + n, d["cols"][1] + at:][:, :dim].double()
            v = d["v"][i * lk:i * lk + n, d["cols"][2] + at:][:, :dim].double()
            p = torch.softmax((q @ k.t() / math.sqrt(dim)).masked_fill(hidden, -math.inf), dim=1)
            out[i, :, j] = torch.where(empty[:, None], torch.zeros((), device="cuda", dtype=torch.float64), p @ v)
    return out.reshape(b * lq, h * dim)
