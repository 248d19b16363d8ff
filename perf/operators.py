"""The 4-bit decode operators of this library, as cases that can be timed and compared.

Four operators carry one decoder block's attention half over weights and a KV
cache that are held in 4 bits: the product of a few rows with 4-bit weights
(``w4``), the norm of every query and key head with the rotary embedding in
the same pass (``qk``), rows into the 4-bit cache and back out of it (``kv4``),
and attention over that cache (``att``).  A case is one such call; the shapes
are those of the repository's decoders (7B-shaped: 32 heads of 128, d 4096,
F 11008; 0.5B-shaped: 14 heads of 64 over 2 KV heads, d 896, F 4864) and
generic grouped-head ones.

``prepare`` builds what a program holds before the call, all from the seed:
activations, 4-bit weights and caches, tables, output buffers and scratch.
``run`` is the call: the plain form in float32, or with ``own`` the library's.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32  # dims that share a scale and a minimum in the cache
EPS = 1e-6


def listed():
    return [
        # the small decoder's O-projection of one token: the launch is most of it
        {"name": "w4_05b_o_b1", "op": "w4", "N": 896, "K": 896, "group": 64, "M": 1, "out": "add", "zeros": False},
        # QKV of one token of the 7B-shaped decoder, the common group size
        {"name": "w4_7b_qkv_b1", "op": "w4", "N": 12288, "K": 4096, "group": 128, "M": 1, "out": "bf16", "zeros": False},
        # its gate/up product with SwiGLU, four sequences, weights with zero points
        {"name": "w4_7b_gateup_b4", "op": "w4", "N": 22016, "K": 4096, "group": 128, "M": 4, "out": "swiglu", "zeros": True},
        # its down product into the residual for an odd batch, the finest groups
        {"name": "w4_7b_down_b13", "op": "w4", "N": 4096, "K": 11008, "group": 32, "M": 13, "out": "add", "zeros": True},
        # queries and keys of a frame of 2048 tokens (1536 visual and 512 text)
        {"name": "qk_7b_2048", "op": "qk", "B": 1, "L": 2048, "H": 32, "Hkv": 32, "dh": 128, "f32": False, "start": 0},
        # one decode step of four sequences from fp32 rows
        {"name": "qk_05b_step_b4", "op": "qk", "B": 4, "L": 1, "H": 14, "Hkv": 2, "dh": 64, "f32": True, "start": 2047},
        # a prefix's keys and values into the cache behind 777 earlier tokens, and out again for a host that continues
        {"name": "kv4_7b_2048", "op": "kv4", "B": 1, "L": 2048, "Hkv": 32, "dh": 128, "start": 777, "ragged": False},
        # the new token of four sequences
        {"name": "kv4_05b_step_b4", "op": "kv4", "B": 4, "L": 1, "Hkv": 2, "dh": 64, "start": 700, "ragged": False},
        # one token of one sequence after a 2048-token frame, a KV head for every head
        {"name": "att_7b_b1_2048", "op": "att", "B": 1, "Lq": 1, "H": 32, "Hkv": 32, "dh": 128, "len": 2049, "ragged": False, "window": 0, "sinks": 0},
        # the small grouped-head decoder, four sequences of different lengths
        {"name": "att_05b_b4_4096", "op": "att", "B": 4, "Lq": 1, "H": 14, "Hkv": 2, "dh": 64, "len": 4097, "ragged": True, "window": 0, "sinks": 0},
        # long contexts, eight sequences: the cache's bytes are everything
        {"name": "att_gqa_b8_32768", "op": "att", "B": 8, "Lq": 1, "H": 32, "Hkv": 8, "dh": 128, "len": 32768, "ragged": True, "window": 0, "sinks": 0},
        # three proposed tokens a sequence, each seeing its last 1024 and the first four tokens
        {"name": "att_window_b16_q3", "op": "att", "B": 16, "Lq": 3, "H": 32, "Hkv": 8, "dh": 128, "len": 8191, "ragged": True, "window": 1024, "sinks": 4},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 32), (14, 2), (32, 8), (16, 16), (8, 1), (28, 4), (40, 8)]


def draw(rng):
    op = rng.choice(["w4", "w4", "w4", "qk", "qk", "kv4", "att", "att", "att"])
    if op == "w4":
        out = rng.choice(["bf16", "f32", "add", "swiglu"])
        K = 8 * _log_int(rng, 32, 1376)
        N = 32 * _log_int(rng, 8, 688) if out == "swiglu" else _log_int(rng, 256, 12288)
        return {"op": "w4", "N": N, "K": K, "group": rng.choice([32, 64, 128]), "M": _log_int(rng, 1, 16), "out": out,
                "zeros": rng.random() < 0.5}
    H, Hkv = rng.choice(HEADS)
    dh = rng.choice([64, 128])
    if op == "qk":
        B = rng.randint(1, 4)
        L = rng.choice([1, _log_int(rng, 2, 2048 // B)])
        return {"op": "qk", "B": B, "L": L, "H": min(H, 32), "Hkv": Hkv if H <= 32 else 32, "dh": dh,
                "f32": rng.random() < 0.3, "start": _log_int(rng, 1, 4096)}
    if op == "kv4":
        B = rng.randint(1, 8)
        L = rng.choice([1, _log_int(rng, 2, 2048 // B)])
        return {"op": "kv4", "B": B, "L": L, "Hkv": Hkv, "dh": dh, "start": _log_int(rng, 1, 4096),
                "ragged": L > 8 and rng.random() < 0.5}
    B = rng.randint(1, 8)
    Lq = rng.choice([1, 1, 1, rng.randint(2, 8)])
    window = rng.choice([0, 0, _log_int(rng, 100, 4096)])
    n = _log_int(rng, 16, 32768 * 8 // max(B * Hkv, 8))
    return {"op": "att", "B": B, "Lq": Lq, "H": H, "Hkv": Hkv, "dh": dh, "len": max(n, Lq), "ragged": rng.random() < 0.5,
            "window": window, "sinks": rng.randint(0, 16) if window else 0}


# ------------------------------------------------------------------- inputs

class _Draws:
    """Seeded tensors on the GPU."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed) % (1 << 62))

    def normal(self, shape, std=1.0, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=self.gen)

    def uniform(self, shape, lo, hi, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda").uniform_(lo, hi, generator=self.gen)

    def ints(self, shape, lo, hi, dtype=torch.uint8):
        return torch.randint(lo, hi, shape, dtype=dtype, device="cuda", generator=self.gen)


def _up(n, m):
    return (n + m - 1) // m * m


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _lens(c):
    """Tokens in each sequence's cache: all alike, or spread from an eighth to the whole."""
    if not c["ragged"] or c["B"] == 1:
        return [c["len"]] * c["B"]
    return [max(c["Lq"], c["len"] - (c["len"] - c["len"] // 8) * b // (c["B"] - 1)) for b in range(c["B"])]


def _counts(c):
    return [c["L"] - (c["L"] * b // (2 * c["B"]) if c["ragged"] else 0) for b in range(c["B"])]


def _rope_tables(n, dh):
    """cos, sin [n][dh/2] in fp32 from angles in fp64."""
    inv = 10000.0 ** (-torch.arange(0, dh, 2, dtype=torch.float64, device="cuda") / dh)
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * inv
    return a.cos().float(), a.sin().float()


def _keys_and_values(c, rnd, n):
    """Projected rows as a decoder leaves them: keys with a few strong channels, values near normal."""
    shape = (c["B"], n, c["Hkv"], c["dh"])
    strong = torch.where(rnd.uniform((c["Hkv"], c["dh"]), 0, 1) < 0.04, 5.0, 1.0) * torch.exp(rnd.normal((c["Hkv"], c["dh"]), 0.3, torch.float32))
    k = (rnd.normal(shape) * strong.bfloat16()).contiguous()
    return k, rnd.normal(shape)


def _inputs(c, seed):
    """The case's inputs as dense arrays, without the library's layouts."""
    rnd = _Draws(seed)
    if c["op"] == "w4":
        G = -(-c["K"] // c["group"])
        s = {"x": rnd.normal((c["M"], c["K"])), "codes": rnd.ints((c["N"], c["K"]), 0, 16),
             "scales": rnd.uniform((c["N"], G), 0.002, 0.01).bfloat16(),
             "zeros": rnd.ints((c["N"], G), 5, 12).bfloat16() if c["zeros"] else None, "residual": None}
        if c["out"] == "add":
            s["residual"] = rnd.normal((c["M"], c["N"]), 1.0, torch.float32)
        return s
    if c["op"] == "qk":
        dt = torch.float32 if c["f32"] else torch.bfloat16
        rows = rnd.normal((c["B"], c["L"], c["H"] + 2 * c["Hkv"], c["dh"]), 1.5, dt)  # the fused projection's rows
        cos, sin = _rope_tables(c["start"] + c["L"] + 3 * c["B"], c["dh"])
        pos = [[c["start"] + 3 * b + t for t in range(c["L"])] for b in range(c["B"])]
        return {"rows": rows, "gq": rnd.uniform((c["dh"],), 0.5, 1.5), "gk": rnd.uniform((c["dh"],), 0.5, 1.5), "cos": cos,
                "sin": sin, "pos": _ints(pos)}
    if c["op"] == "kv4":
        k, v = _keys_and_values(c, rnd, c["L"])
        return {"k": k, "v": v, "start": _ints([c["start"] + 5 * b for b in range(c["B"])]), "count": _ints(_counts(c))}
    k, v = _keys_and_values(c, rnd, c["len"])
    q = rnd.normal((c["B"], c["Lq"], c["H"], c["dh"]))
    return {"k": k, "v": v, "q": q, "lens": _ints(_lens(c))}


def _cap(c):
    """Rows of the cache: a multiple of 32, with room for what comes next."""
    n = c["start"] + 5 * c["B"] + c["L"] if c["op"] == "kv4" else c["len"]
    return _up(n + 1, 32)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    dev = dict(device="cuda")
    if case["op"] == "w4":
        wide = case["N"] // 2 if case["out"] == "swiglu" else case["N"]
        s["y"] = torch.empty((case["M"], wide), dtype=torch.float32 if case["out"] in ("f32", "add") else torch.bfloat16, **dev)
        if own:  # the weights as a program holds them: packed once, at load
            from paper_2608_14586_amd import binding as vb
            packed = torch.empty(vb.vla_op_w4_packed_bytes(case["N"], case["K"], case["group"]), dtype=torch.uint8, **dev)
            vb.vla_op_w4_pack(s.pop("codes"), s.pop("scales"), s.pop("zeros"), packed, case["group"])
            s["packed"] = packed
        return s
    if case["op"] == "qk":
        H, Hkv = case["H"], case["Hkv"]
        s["q"], s["k"] = s["rows"][:, :, :H], s["rows"][:, :, H:H + Hkv]
        s["q_out"] = torch.empty((case["B"], case["L"], H, case["dh"]), dtype=torch.bfloat16, **dev)
        s["k_out"] = torch.empty((case["B"], case["L"], Hkv, case["dh"]), dtype=torch.bfloat16, **dev)
        return s
    if case["op"] == "kv4":
        s["k_out"], s["v_out"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        s["cap"] = _cap(case)
        if own:
            from paper_2608_14586_amd import binding as vb
            s["cache"] = torch.zeros(vb.vla_op_kv4_bytes(case["B"], case["Hkv"], s["cap"], case["dh"]), dtype=torch.uint8, **dev)
        else:
            s["cache"] = _Cache(case["B"], s["cap"], case["Hkv"], case["dh"])
        return s
    k, v = s.pop("k"), s.pop("v")
    s["cap"], s["max_len"] = _cap(case), max(_lens(case))
    s["o"] = torch.empty_like(s["q"])
    if own:
        from paper_2608_14586_amd import binding as vb
        s["cache"] = torch.zeros(vb.vla_op_kv4_bytes(case["B"], case["Hkv"], s["cap"], case["dh"]), dtype=torch.uint8, **dev)
        vb.vla_op_kv4_store(k, v, None, s["lens"], s["cache"], s["cap"])
        s["scratch"] = torch.empty(vb.vla_op_attention_kv4_scratch(case["B"], case["Lq"], case["H"], case["Hkv"], case["dh"],
                                                                   s["max_len"], case["window"], case["sinks"]), dtype=torch.uint8, **dev)
    else:
        s["kq"], s["vq"] = _quantise(k), _quantise(v)
    return s


# -------------------------------------------------------------- plain forms

def _quantise(x):
    """(codes, scale, minimum) of rows x [..., dh] in groups of 32 dims: scale =
    (max - min) / 15 in bf16, code = (x - min) / scale to the nearest, ties to
    the even one, at most 15."""
    g = x.unflatten(-1, (-1, GROUP)).float()
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    scale = ((hi - lo) / 15).bfloat16().float()
    codes = torch.where(scale > 0, (g - lo) / scale, torch.zeros_like(g)).round().clamp_max(15)
    return codes.to(torch.uint8), scale.bfloat16(), lo.bfloat16()


def _values(q):
    codes, scale, lo = q
    return (codes.float() * scale.float() + lo.float()).flatten(-2)


class _Cache:
    """Codes, scales and minimums of keys and values, [B][cap][Hkv][dh / 32][...]."""

    def __init__(self, B, cap, Hkv, dh):
        shape = (2, B, cap, Hkv, dh // GROUP)
        self.codes = torch.zeros(shape + (GROUP,), dtype=torch.uint8, device="cuda")
        self.scale = torch.zeros(shape + (1,), dtype=torch.bfloat16, device="cuda")
        self.lo = torch.zeros(shape + (1,), dtype=torch.bfloat16, device="cuda")


def _plain_w4(s):
    c = s["case"]
    N, K, g = c["N"], c["K"], c["group"]
    scale = s["scales"].float().repeat_interleave(g, 1)[:, :K]
    zero = 8.0 if s["zeros"] is None else s["zeros"].float().repeat_interleave(g, 1)[:, :K]
    y = s["x"].float() @ ((s["codes"].float() - zero) * scale).T
    if c["out"] == "add":
        return y + s["residual"]
    if c["out"] == "f32":
        return y
    if c["out"] == "swiglu":
        gate, up = y[:, :N // 2], y[:, N // 2:]
        y = gate / (1 + torch.exp(-gate)) * up
    return y.bfloat16()


def _plain_head(x, gain, cos, sin):
    x = x.float()
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).bfloat16()


def _plain_qk(s):
    at = s["pos"].long()
    cos, sin = s["cos"][at][:, :, None], s["sin"][at][:, :, None]
    return _plain_head(s["q"], s["gq"], cos, sin), _plain_head(s["k"], s["gk"], cos, sin)


def _plain_kv4(s):
    c, cache = s["case"], s["cache"]
    t = torch.arange(c["L"], device="cuda")
    b = torch.arange(c["B"], device="cuda")[:, None].expand(-1, c["L"])
    at = s["start"].long()[:, None] + t
    there = (t < s["count"][:, None])[..., None, None]
    new = [torch.stack(x) for x in zip(_quantise(s["k"]), _quantise(s["v"]))]
    old = [cache.codes[:, b, at], cache.scale[:, b, at], cache.lo[:, b, at]]
    cache.codes[:, b, at] = torch.where(there[..., None], new[0], old[0])
    cache.scale[:, b, at] = torch.where(there[..., None], new[1], old[1])
    cache.lo[:, b, at] = torch.where(there[..., None], new[2], old[2])
    back = _values((cache.codes[:, b, at], cache.scale[:, b, at], cache.lo[:, b, at])).bfloat16()
    return torch.where(there, back[0], s["k_out"]), torch.where(there, back[1], s["v_out"])


def _seen(c, lens, n):
    """(positions [B][n'], whether query i of sequence b sees each [B][Lq][n'])
    over the n cached tokens, or over the first tokens and the last ones where
    a window leaves fewer."""
    Lq, window, sinks = c["Lq"], c["window"], c["sinks"]
    at = torch.arange(n, device="cuda").expand(c["B"], -1)
    span = window + Lq - 1
    if window and sinks + span < n:
        first = (lens - span).clamp(sinks, n - span)[:, None]
        at = torch.cat([at[:, :sinks], first + at[:, :span]], 1)
    q = (lens[:, None] - Lq + torch.arange(Lq, device="cuda"))[:, :, None]
    key = at[:, None, :]
    sees = key <= q
    if window:
        sees = sees & ((key > q - window) | (key < sinks))
    return at, sees


def _plain_att(s):
    c = s["case"]
    G = c["H"] // c["Hkv"]
    at, sees = _seen(c, s["lens"].long(), s["max_len"])
    b = torch.arange(c["B"], device="cuda")[:, None]
    whole = at.shape[1] == s["max_len"]
    k, v = (_values(x if whole else tuple(part[b, at] for part in x)).transpose(1, 2).contiguous() for x in (s["kq"], s["vq"]))
    q = s["q"].float().unflatten(2, (c["Hkv"], G)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [B][Hkv][Lq G][dh]
    p = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (1 / math.sqrt(c["dh"]))
    p = p.unflatten(2, (c["Lq"], G)).masked_fill_(~sees[:, None, :, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p = torch.exp(p - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (c["Lq"], G)) / torch.where(total == 0, torch.ones_like(total), total)
    return o.permute(0, 2, 1, 3, 4).flatten(2, 3).bfloat16()


def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    return {"w4": _plain_w4, "qk": _plain_qk, "kv4": _plain_kv4, "att": _plain_att}[op](state)


# ------------------------------------------------------- the library's calls

def _own_w4(s):
    from paper_2608_14586_amd import binding as vb
    c = s["case"]
    vb.vla_op_gemv_w4(s["x"], s["packed"], s["residual"], s["y"], c["N"], c["group"], c["out"] == "swiglu")
    return s["y"]


def _own_qk(s):
    from paper_2608_14586_amd import binding as vb
    vb.vla_op_qk_norm_rope(s["q"], s["k"], s["gq"], s["gk"], EPS, s["cos"], s["sin"], s["pos"], s["q_out"], s["k_out"])
    return s["q_out"], s["k_out"]


def _own_kv4(s):
    from paper_2608_14586_amd import binding as vb
    vb.vla_op_kv4_store(s["k"], s["v"], s["start"], s["count"], s["cache"], s["cap"])
    vb.vla_op_kv4_load(s["cache"], s["cap"], s["start"], s["count"], s["k_out"], s["v_out"])
    return s["k_out"], s["v_out"]


def _own_att(s):
    from paper_2608_14586_amd import binding as vb
    c = s["case"]
    vb.vla_op_attention_kv4(s["q"], s["cache"], s["cap"], c["Hkv"], s["lens"], s["o"], s["max_len"], c["window"], c["sinks"], s["scratch"])
    return s["o"]


_OWN = {"w4": _own_w4, "qk": _own_qk, "kv4": _own_kv4, "att": _own_att}


# ------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "w4":
        G = -(-c["K"] // c["group"])
        wide = c["N"] // 2 if c["out"] == "swiglu" else c["N"]
        width = {"bf16": 2, "swiglu": 2, "f32": 4, "add": 8}[c["out"]]
        read = c["N"] * c["K"] / 2 + c["N"] * G * (4 if c["zeros"] else 2) + c["M"] * c["K"] * 2
        return {"bytes": read + c["M"] * wide * width, "flops": 2 * c["M"] * c["N"] * c["K"]}
    if c["op"] == "qk":
        n = c["B"] * c["L"] * (c["H"] + c["Hkv"]) * c["dh"]
        return {"bytes": n * ((4 if c["f32"] else 2) + 2) + c["B"] * c["L"] * (c["dh"] * 4 + 4), "flops": 9 * n}
    row = c["dh"] // 2 + c["dh"] // GROUP * 4  # a cached key or value
    if c["op"] == "kv4":
        n = 2 * sum(_counts(c)) * c["Hkv"]
        return {"bytes": n * (2 * row + 4 * c["dh"]), "flops": 8 * n * c["dh"]}
    Lq, window, sinks = c["Lq"], c["window"], c["sinks"]
    keys, pairs = 0, 0
    for n in _lens(c):
        keys += min(n, sinks + window + Lq - 1) if window else n
        for i in range(Lq):
            m = n - Lq + i + 1
            pairs += min(m, window) + min(sinks, max(m - window, 0)) if window else m
    return {"bytes": keys * c["Hkv"] * 2 * row + c["B"] * Lq * c["H"] * c["dh"] * 4, "flops": 4 * pairs * c["H"] * c["dh"]}


# ------------------------------------------------------------ the definitions in 64 bits

def _exact_groups(x):
    """The values that x [..., dh] has in the cache."""
    g = x.double().reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    lo = g.min(-1, keepdim=True).values
    step = ((g.max(-1, keepdim=True).values - lo) / 15).to(torch.bfloat16).double()
    code = torch.round((g - lo) / step.clamp_min(1e-300)).clamp(0, 15) * (step > 0)
    return (lo + code * step).reshape(x.shape)


def _exact_w4(c, s):
    group = torch.arange(c["K"], device="cuda") // c["group"]
    zero = s["zeros"].double()[:, group] if s["zeros"] is not None else 8
    w = s["scales"].double()[:, group] * (s["codes"].double() - zero)
    y = torch.mm(s["x"].double(), w.t().contiguous())
    if c["out"] == "swiglu":
        half = c["N"] // 2
        return y[:, :half] * torch.sigmoid(y[:, :half]) * y[:, half:]
    return y + s["residual"].double() if c["out"] == "add" else y


def _exact_qk(c, s):
    out = []
    half = c["dh"] // 2
    for first, n, gain in ((0, c["H"], s["gq"]), (c["H"], c["Hkv"], s["gk"])):
        x = s["rows"][:, :, first:first + n].double()
        y = gain.double() * x * torch.rsqrt(x.pow(2).sum(-1, keepdim=True) / c["dh"] + EPS)
        # the pair (i, i + dh/2) as one complex number, turned by its angle
        turn = torch.complex(s["cos"].double(), s["sin"].double())[s["pos"].long()].unsqueeze(2)
        z = torch.complex(y[..., :half].contiguous(), y[..., half:].contiguous()) * turn
        out.append(torch.cat([z.real, z.imag], -1))
    return tuple(out)


def _exact_kv4(c, s):
    out = []
    for x in (s["k"], s["v"]):
        y = _exact_groups(x)
        for b, n in enumerate(_counts(c)):
            y[b, n:] = 0
        out.append(y)
    return tuple(out)


def _exact_att(c, s):
    G, Lq = c["H"] // c["Hkv"], c["Lq"]
    o = torch.zeros((c["B"], Lq, c["H"], c["dh"]), dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lens(c)):
        lo = max(0, n - c["window"] - Lq + 1) if c["window"] else 0
        keep = [j for j in range(min(c["sinks"], lo))] + list(range(lo, n))
        at = torch.tensor(keep, device="cuda")
        k, v = _exact_groups(s["k"][b, at]), _exact_groups(s["v"][b, at])
        for i in range(Lq):
            me = n - Lq + i
            hidden = at > me
            if c["window"]:
                hidden = hidden | ((me - at >= c["window"]) & (at >= c["sinks"]))
            for h in range(c["Hkv"]):
                w = s["q"][b, i, h * G:(h + 1) * G].double() @ k[:, h].t().contiguous() / math.sqrt(c["dh"])
                w[:, hidden] = -math.inf
                o[b, i, h * G:(h + 1) * G] = torch.softmax(w, -1) @ v[:, h].contiguous()
    return o


def exact(case, seed):
    s = _inputs(case, seed)
    return {"w4": _exact_w4, "qk": _exact_qk, "kv4": _exact_kv4, "att": _exact_att}[case["op"]](case, s)
