"""The 8-bit and packed-prompt operators of this library, as cases that can be
timed and compared.

They carry a decoder block over prompts of different lengths with 8-bit
weights, activations and cache, and the decode steps that follow: RMS norm with
the residual's addition into int8 rows with a scale each (``norm``; without a
gain, rows into int8), the product of int8 rows with int8 weights (``gemm``),
causal attention over packed prompts (``pack``), rows into the 8-bit cache and
back out of it (``kv8``), and attention over that cache (``att``).  A case is one
such call; the shapes are those of the repository's decoders (7B-shaped: 32
heads of 128, d 4096, F 11008; 0.5B-shaped: 14 heads of 64 over 2 KV heads, d
896, F 4864) and generic grouped-head ones.

``prepare`` builds what a program holds before the call, all from the seed.
``run`` is the call: the plain form in float32, or with ``own`` the library's.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32  # positions of a head that share a scale in the cache
EPS = 1e-6


def listed():
    return [
        # the attention half's norm of one step of four sequences of the small decoder: the launch is most of it
        {"name": "norm_05b_step_b4", "op": "norm", "M": 4, "d": 896, "x": "f32", "add": "f32", "norm": True},
        # the MLP's norm over a frame of 2048 tokens, behind the attention half's bf16 output
        {"name": "norm_7b_2048", "op": "norm", "M": 2048, "d": 4096, "x": "f32", "add": "bf16", "norm": True},
        # the gated activation of an odd number of tokens on its way into the down product
        {"name": "norm_7b_rows_1777", "op": "norm", "M": 1777, "d": 11008, "x": "bf16", "add": "", "norm": False},
        # QKV of one token: the weights' bytes are everything
        {"name": "gemm_7b_qkv_b1", "op": "gemm", "M": 1, "N": 12288, "K": 4096, "out": "bf16"},
        # down product into the residual for a short prompt of odd length
        {"name": "gemm_7b_down_333", "op": "gemm", "M": 333, "N": 4096, "K": 11008, "out": "add"},
        # gate/up product with SwiGLU over a frame of 2048 tokens: the matrix cores
        {"name": "gemm_7b_gateup_2048", "op": "gemm", "M": 2048, "N": 22016, "K": 4096, "out": "swiglu"},
        # nine short prompts of the small decoder, one of a single token, rows of padding behind them
        {"name": "pack_05b_9", "op": "pack", "H": 14, "Hkv": 2, "dh": 64, "lens": "701,64,1,333,128,417,95,256,29", "pad": 24},
        # a long prompt, a frame and two shorter ones of the 7B-shaped decoder
        {"name": "pack_7b_4", "op": "pack", "H": 32, "Hkv": 32, "dh": 128, "lens": "4096,2048,1201,847", "pad": 0},
        # a frame's keys and values into the cache behind 777 earlier tokens, and out again for a host that continues
        {"name": "kv8_7b_2048", "op": "kv8", "B": 1, "L": 2048, "Hkv": 32, "dh": 128, "start": 777, "ragged": False},
        # the new token of four sequences
        {"name": "kv8_05b_step_b4", "op": "kv8", "B": 4, "L": 1, "Hkv": 2, "dh": 64, "start": 700, "ragged": False},
        # one token of one sequence after a 2048-token frame, a KV head for every head
        {"name": "att_7b_b1_2048", "op": "att", "B": 1, "Lq": 1, "H": 32, "Hkv": 32, "dh": 128, "len": 2049, "ragged": False, "window": 0, "sinks": 0},
        # long contexts, eight sequences: the cache's bytes are everything
        {"name": "att_gqa_b8_32768", "op": "att", "B": 8, "Lq": 1, "H": 32, "Hkv": 8, "dh": 128, "len": 32768, "ragged": True, "window": 0, "sinks": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 32), (14, 2), (32, 8), (16, 16), (8, 1), (28, 4), (40, 8)]


def draw(rng):
    op = rng.choice(["norm", "gemm", "gemm", "gemm", "pack", "pack", "kv8", "att", "att"])
    if op == "norm":
        norm = rng.random() < 0.6
        return {"op": "norm", "M": _log_int(rng, 1, 2048), "d": 8 * _log_int(rng, 16, 1024 if norm else 1376),
                "x": "f32" if norm else rng.choice(["bf16", "f32"]), "add": rng.choice(["", "bf16", "f32"]) if norm else "",
                "norm": norm}
    if op == "gemm":
        out = rng.choice(["bf16", "f32", "add", "swiglu"])
        K = 16 * _log_int(rng, 16, 688)
        N = 64 * _log_int(rng, 4, 344) if out == "swiglu" else _log_int(rng, 256, 12288)
        M = rng.choice([rng.randint(1, 16), _log_int(rng, 17, max(18, min(4096, 180_000_000_000 // (N * K))))])
        return {"op": "gemm", "M": M, "N": N, "K": K, "out": out}
    H, Hkv = rng.choice(HEADS)
    dh = rng.choice([64, 128])
    if op == "pack":
        lens, tokens, pairs = [], 8192, 11_500_000 * 32 // max(H, 32)
        for _ in range(rng.randint(1, 12)):
            n = rng.choice([_log_int(rng, 1, 4096), _log_int(rng, 16, 512)])
            if n <= tokens and n * (n + 1) // 2 <= pairs:
                lens.append(n)
                tokens -= n
                pairs -= n * (n + 1) // 2
        return {"op": "pack", "H": H, "Hkv": Hkv, "dh": dh, "lens": ",".join(map(str, lens or [77])), "pad": rng.choice([0, rng.randint(1, 40)])}
    if op == "kv8":
        B = rng.randint(1, 8)
        L = rng.choice([1, _log_int(rng, 2, 2048 // B)])
        return {"op": "kv8", "B": B, "L": L, "Hkv": Hkv, "dh": dh, "start": _log_int(rng, 1, 4096),
                "ragged": L > 8 and rng.random() < 0.5}
    B = rng.randint(1, 8)
    Lq = rng.choice([1, 1, 1, rng.randint(2, 8)])
    window = rng.choice([0, 0, _log_int(rng, 100, 4096)])
    n = _log_int(rng, 16, 32768 * 64 // max(B * Hkv, 64))
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


DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


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


def _starts(c):
    return [c["start"] + 5 * b for b in range(c["B"])]


def _ahead(c):
    """Rows ahead of the stored ones that are read back with them: those of a block that the stored ones may rescale."""
    return min(c["start"], BLOCK - 1)


def _prompts(c):
    """Offsets of the packed prompts."""
    at = [0]
    for n in c["lens"].split(","):
        at.append(at[-1] + int(n))
    return at


def _hidden(rnd, shape, dtype):
    """Rows of a residual stream: near normal, a few channels far larger."""
    strong = torch.where(rnd.uniform((shape[-1],), 0, 1) < 0.005, 20.0, 1.0)
    return (rnd.normal(shape, 1.0, torch.float32) * strong).to(dtype)


def _codes(rnd, shape):
    """Rows as quantisers leave them: near normal, the largest at 127."""
    return rnd.normal(shape, 36.0, torch.float32).round_().clamp_(-127, 127).to(torch.int8)


def _keys_and_values(c, rnd, n):
    """Projected rows as a decoder leaves them: keys with a few strong channels, values near normal."""
    shape = (c["B"], n, c["Hkv"], c["dh"])
    strong = torch.where(rnd.uniform((c["Hkv"], c["dh"]), 0, 1) < 0.04, 5.0, 1.0) * torch.exp(rnd.normal((c["Hkv"], c["dh"]), 0.3, torch.float32))
    k = (rnd.normal(shape) * strong.bfloat16()).contiguous()
    return k, rnd.normal(shape)


def _inputs(c, seed):
    """The case's inputs as dense arrays, without the library's layouts."""
    rnd = _Draws(seed)
    if c["op"] == "norm":
        shape = (c["M"], c["d"])
        return {"x": _hidden(rnd, shape, DTYPE[c["x"]]), "add": _hidden(rnd, shape, DTYPE[c["add"]]) if c["add"] else None,
                "g": rnd.uniform((c["d"],), 0.5, 1.5) if c["norm"] else None}
    if c["op"] == "gemm":
        wide = c["N"] // 2 if c["out"] == "swiglu" else c["N"]
        size = 1 / (36.0 * 36.0 * math.sqrt(c["K"]))  # results near one
        return {"x": _codes(rnd, (c["M"], c["K"])), "sx": rnd.uniform((c["M"],), 0.5, 2.0), "w": _codes(rnd, (c["N"], c["K"])),
                "sw": rnd.uniform((c["N"],), 0.5 * size, 2.0 * size),
                "residual": rnd.normal((c["M"], wide), 1.0, torch.float32) if c["out"] == "add" else None}
    if c["op"] == "pack":
        at = _prompts(c)
        # the fused projection's rows
        rows = rnd.normal((at[-1] + c["pad"], c["H"] + 2 * c["Hkv"], c["dh"]))
        return {"rows": rows, "offsets": _ints(at)}
    if c["op"] == "kv8":
        k0, v0 = _keys_and_values(c, rnd, max(_starts(c)))
        k, v = _keys_and_values(c, rnd, c["L"])
        return {"k0": k0, "v0": v0, "k": k, "v": v, "start": _ints(_starts(c)), "count": _ints(_counts(c))}
    k, v = _keys_and_values(c, rnd, c["len"])
    q = rnd.normal((c["B"], c["Lq"], c["H"], c["dh"]))
    return {"k": k, "v": v, "q": q, "lens": _ints(_lens(c))}


def _cap(c):
    """Rows of the cache: a multiple of 32, with room for what comes next."""
    n = max(_starts(c)) + c["L"] if c["op"] == "kv8" else c["len"]
    return _up(n + 1, 32)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    dev = dict(device="cuda")
    if case["op"] == "norm":
        M, d = case["M"], case["d"]
        s["sum"] = torch.empty((M, d), **dev) if case["add"] else None
        s["codes"], s["scales"] = torch.empty((M, d), dtype=torch.int8, **dev), torch.empty(M, **dev)
        return s
    if case["op"] == "gemm":
        wide = case["N"] // 2 if case["out"] == "swiglu" else case["N"]
        s["y"] = torch.empty((case["M"], wide), dtype=torch.float32 if case["out"] in ("f32", "add") else torch.bfloat16, **dev)
        if own:  # the weights as a program holds them: packed once, at load
            from paper_2608_14586_amd import binding as vb
            s["packed"] = torch.empty(vb.vla_op_w8_packed_bytes(case["N"], case["K"]), dtype=torch.uint8, **dev)
            vb.vla_op_w8_pack(s.pop("w"), s.pop("sw"), s["packed"])
        return s
    if case["op"] == "pack":
        H, Hkv = case["H"], case["Hkv"]
        s["q"], s["k"], s["v"] = s["rows"][:, :H], s["rows"][:, H:H + Hkv], s["rows"][:, H + Hkv:]
        s["o"] = torch.zeros((s["rows"].shape[0], H, case["dh"]), dtype=torch.bfloat16, **dev)
        return s
    if case["op"] == "kv8":
        k0, v0 = s.pop("k0"), s.pop("v0")
        ahead = _ahead(case)
        shape = (case["B"], case["L"] + ahead, case["Hkv"], case["dh"])
        s["k_out"], s["v_out"] = (torch.zeros(shape, dtype=torch.bfloat16, **dev) for _ in range(2))
        s["from"], s["n_out"], s["cap"] = s["start"] - ahead, s["count"] + ahead, _cap(case)
        if own:
            from paper_2608_14586_amd import binding as vb
            s["cache"] = torch.zeros(vb.vla_op_kv8_bytes(case["B"], case["Hkv"], s["cap"], case["dh"]), dtype=torch.uint8, **dev)
            vb.vla_op_kv8_store(k0, v0, None, s["start"], s["cache"], s["cap"])
        else:
            s["cache"] = [_Cache(x, s["start"], s["cap"]) for x in (k0, v0)]
        return s
    k, v = s.pop("k"), s.pop("v")
    s["cap"], s["max_len"] = _cap(case), max(_lens(case))
    s["o"] = torch.empty_like(s["q"])
    if own:
        from paper_2608_14586_amd import binding as vb
        s["cache"] = torch.zeros(vb.vla_op_kv8_bytes(case["B"], case["Hkv"], s["cap"], case["dh"]), dtype=torch.uint8, **dev)
        vb.vla_op_kv8_store(k, v, None, s["lens"], s["cache"], s["cap"])
        s["scratch"] = torch.empty(vb.vla_op_attention_kv8_scratch(case["B"], case["Lq"], case["H"], case["Hkv"], case["dh"],
                                                                   s["max_len"], case["window"], case["sinks"]), dtype=torch.uint8, **dev)
    else:
        s["kq"], s["vq"] = (_Cache(x, s["lens"], s["cap"]) for x in (k, v))
    return s


# -------------------------------------------------------------- plain forms

def _plain_norm(s):
    c = s["case"]
    t = s["x"].float()
    if c["add"]:
        t = t + s["add"].float()
    u = t * s["g"] if c["norm"] else t
    top = u.abs().amax(-1, keepdim=True)
    code = torch.round(127 * u.double() / top.double()).float()  # next to a border between two codes 32 bits are too few
    step = top / 127
    if c["norm"]:
        step = step / torch.sqrt((t * t).mean(-1, keepdim=True) + EPS)
    return ((t,) if c["add"] else ()) + (code * step, step[:, 0])


def _plain_gemm(s):
    c = s["case"]
    y = (s["x"].float() @ s["w"].float().T) * s["sx"][:, None] * s["sw"]
    if c["out"] == "add":
        return y + s["residual"]
    if c["out"] == "f32":
        return y
    if c["out"] == "swiglu":
        gate, up = y.chunk(2, -1)
        y = gate / (1 + torch.exp(-gate)) * up
    return y.bfloat16()


def _softmax_product(q, k, v, sees):
    """softmax(q k^T / sqrt(dh)) v over the keys that each query sees; zeros where it sees none."""
    p = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (1 / math.sqrt(q.shape[-1]))
    p = p.masked_fill_(~sees, -math.inf)
    top = p.amax(-1, keepdim=True)
    p = torch.exp(p - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)


def _plain_pack(s):
    c, o = s["case"], s["o"]
    G = c["H"] // c["Hkv"]
    at = _prompts(c)
    for a, b in zip(at, at[1:]):
        t = torch.arange(b - a, device="cuda")
        sees = t <= t[:, None]
        q, k, v = (s[x][a:b].float().transpose(0, 1).contiguous() for x in ("q", "k", "v"))
        for h in range(c["Hkv"]):  # one KV head's scores at a time
            y = _softmax_product(q[h * G:(h + 1) * G], k[h].expand(G, -1, -1), v[h].expand(G, -1, -1), sees)
            o[a:b, h * G:(h + 1) * G] = y.transpose(0, 1).bfloat16()
    return o


def _fp8_step(x):
    """The smallest power of two that takes the largest of |x| over its last dimensions to 448 or less."""
    m, e = torch.frexp(x)
    e = e - 9 + (m > 0.875).int()
    return torch.ldexp(torch.ones_like(x), torch.where(x > 0, e, torch.full_like(e, -118)).clamp_min(-118))


class _Cache:
    """Codes [B][cap / 32][32][Hkv][dh] of keys or of values, and steps [B][cap / 32][1][Hkv][1]."""

    def __init__(self, x, count, cap):
        B, L, Hkv, dh = x.shape
        self.codes = torch.zeros((B, cap // BLOCK, BLOCK, Hkv, dh), dtype=torch.uint8, device="cuda")
        self.step = torch.full((B, cap // BLOCK, 1, Hkv, 1), 2.0 ** -118, device="cuda")
        self.store(x, torch.zeros(B, dtype=torch.long, device="cuda"), count)

    def store(self, x, start, count):
        B, L, Hkv, dh = x.shape
        nb = min((L + 2 * (BLOCK - 1)) // BLOCK, self.codes.shape[1])
        first = (start.long() // BLOCK).clamp_max(self.codes.shape[1] - nb)
        at = first[:, None] + torch.arange(nb, device="cuda")
        b = torch.arange(B, device="cuda")[:, None]
        pos = (at[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten(1) - start[:, None]
        here = (pos >= 0) & (pos < count[:, None])
        new = torch.where(here[..., None, None], x[b, pos.clamp(0, L - 1)].float(), 0.0).unflatten(1, (nb, BLOCK))
        here = here.unflatten(1, (nb, BLOCK))[..., None, None]
        step, codes = self.step[b, at], self.codes[b, at].view(torch.float8_e4m3fn)
        need = _fp8_step(new.abs().amax((2, 4), keepdim=True))
        anew = here[:, :, :1]  # the block's first row is stored: it begins again
        grown = torch.where(anew, need, torch.maximum(step, need))
        grown = torch.where(here.any(2, keepdim=True), grown, step)
        old = codes.float() * torch.where(anew, torch.ones_like(step), step / grown)
        self.codes[b, at] = torch.where(here, new / grown, old).to(torch.float8_e4m3fn).view(torch.uint8)
        self.step[b, at] = grown

    def values(self, b, at):
        return self.codes[b, at // BLOCK, at % BLOCK].view(torch.float8_e4m3fn).float() * self.step[b, at // BLOCK, 0]

    def all(self, n):
        return (self.codes.view(torch.float8_e4m3fn).float() * self.step).flatten(1, 2)[:, :n]


def _plain_kv8(s):
    b = torch.arange(s["k"].shape[0], device="cuda")[:, None]
    t = torch.arange(s["k_out"].shape[1], device="cuda")
    at = s["from"].long()[:, None] + t
    there = (t < s["n_out"][:, None])[..., None, None]
    out = []
    for cache, x, old in zip(s["cache"], (s["k"], s["v"]), (s["k_out"], s["v_out"])):
        cache.store(x, s["start"], s["count"])
        out.append(torch.where(there, cache.values(b, at).bfloat16(), old))
    return tuple(out)


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
    n = s["max_len"]
    at, sees = _seen(c, s["lens"].long(), n)
    b = torch.arange(c["B"], device="cuda")[:, None]
    k, v = ((x.all(n) if at.shape[1] == n else x.values(b, at)).transpose(1, 2).contiguous() for x in (s["kq"], s["vq"]))
    q = s["q"].float().unflatten(2, (c["Hkv"], G)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [B][Hkv][Lq G][dh]
    o = _softmax_product(q, k, v, sees.repeat_interleave(G, 1)[:, None])
    return o.unflatten(2, (c["Lq"], G)).permute(0, 2, 1, 3, 4).flatten(2, 3).bfloat16()


def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    return {"norm": _plain_norm, "gemm": _plain_gemm, "pack": _plain_pack, "kv8": _plain_kv8, "att": _plain_att}[op](state)


# ------------------------------------------------------- the library's calls

def _own_norm(s):
    from paper_2608_14586_amd import binding as vb
    vb.vla_op_norm_i8(s["x"], s["add"], s["sum"], s["g"], EPS, s["codes"], s["scales"])
    return ((s["sum"],) if s["case"]["add"] else ()) + (s["codes"] * s["scales"][:, None], s["scales"])


def _own_gemm(s):
    from paper_2608_14586_amd import binding as vb
    c = s["case"]
    vb.vla_op_gemm_i8(s["x"], s["sx"], s["packed"], s["residual"], s["y"], c["N"], c["out"] == "swiglu")
    return s["y"]


def _own_pack(s):
    from paper_2608_14586_amd import binding as vb
    vb.vla_op_attention_packed(s["q"], s["k"], s["v"], s["offsets"], s["o"])
    return s["o"]


def _own_kv8(s):
    from paper_2608_14586_amd import binding as vb
    vb.vla_op_kv8_store(s["k"], s["v"], s["start"], s["count"], s["cache"], s["cap"])
    vb.vla_op_kv8_load(s["cache"], s["cap"], s["from"], s["n_out"], s["k_out"], s["v_out"])
    return s["k_out"], s["v_out"]


def _own_att(s):
    from paper_2608_14586_amd import binding as vb
    c = s["case"]
    vb.vla_op_attention_kv8(s["q"], s["cache"], s["cap"], c["Hkv"], s["lens"], s["o"], s["max_len"], c["window"], c["sinks"], s["scratch"])
    return s["o"]


_OWN = {"norm": _own_norm, "gemm": _own_gemm, "pack": _own_pack, "kv8": _own_kv8, "att": _own_att}


# ------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "norm":
        n = c["M"] * c["d"]
        width = {"": 0, "f32": 4, "bf16": 2}
        read = width[c["x"]] + width[c["add"]] + (4 if c["add"] else 0)
        return {"bytes": n * (read + 1) + c["M"] * 4 + c["d"] * 4 * c["norm"], "flops": 6 * n}
    if c["op"] == "gemm":
        wide = c["N"] // 2 if c["out"] == "swiglu" else c["N"]
        width = {"bf16": 2, "swiglu": 2, "f32": 4, "add": 8}[c["out"]]
        return {"bytes": (c["N"] + c["M"]) * (c["K"] + 4) + c["M"] * wide * width, "flops": 2 * c["M"] * c["N"] * c["K"]}
    if c["op"] == "pack":
        at = _prompts(c)
        pairs = sum((b - a) * (b - a + 1) // 2 for a, b in zip(at, at[1:]))
        return {"bytes": at[-1] * (2 * c["H"] + 2 * c["Hkv"]) * c["dh"] * 2 + 4 * len(at), "flops": 4 * pairs * c["H"] * c["dh"]}
    row = c["dh"] + 4 / BLOCK  # a cached key or value
    if c["op"] == "kv8":
        n, ahead = 2 * sum(_counts(c)) * c["Hkv"], 2 * c["B"] * _ahead(c) * c["Hkv"]
        return {"bytes": n * (2 * row + 4 * c["dh"]) + ahead * (row + 2 * c["dh"]), "flops": 4 * n * c["dh"]}
    Lq, window, sinks = c["Lq"], c["window"], c["sinks"]
    keys, pairs = 0, 0
    for n in _lens(c):
        keys += min(n, sinks + window + Lq - 1) if window else n
        for i in range(Lq):
            m = n - Lq + i + 1
            pairs += min(m, window) + min(sinks, max(m - window, 0)) if window else m
    return {"bytes": keys * c["Hkv"] * 2 * row + c["B"] * Lq * c["H"] * c["dh"] * 4, "flops": 4 * pairs * c["H"] * c["dh"]}


# ------------------------------------------------------------ the definitions in 64 bits

def _held(x):
    """As 32 bits hold it: the sum is, and its product with the gain, before codes are chosen."""
    return x.to(torch.float32).to(torch.float64)


def _exact_norm(c, s):
    x = s["x"].double()
    y = x if s["add"] is None else _held(x + s["add"].double())
    z = y if s["g"] is None else _held(y * s["g"].double())
    top = z.abs().max(-1, keepdim=True).values
    code = torch.round(127 * z / top)
    scale = top / 127
    if s["g"] is not None:
        scale = scale * torch.rsqrt(y.pow(2).sum(-1, keepdim=True) / c["d"] + EPS)
    return (() if s["add"] is None else (y,)) + (code * scale, scale.squeeze(-1))


def _exact_gemm(c, s):
    y = torch.mm(s["x"].double(), s["w"].double().t().contiguous())  # whole numbers below 2^53
    y = y * (s["sx"].double()[:, None] * s["sw"].double()[None])
    if c["out"] == "swiglu":
        half = c["N"] // 2
        return y[:, :half] * torch.sigmoid(y[:, :half]) * y[:, half:]
    return y + s["residual"].double() if c["out"] == "add" else y


def _exact_pack(c, s):
    H, Hkv = c["H"], c["Hkv"]
    o = torch.zeros((s["rows"].shape[0], H, c["dh"]), dtype=torch.float64, device="cuda")
    at = _prompts(c)
    for a, b in zip(at[:-1], at[1:]):
        later = torch.ones((b - a, b - a), dtype=torch.bool, device="cuda").triu(1)
        for h in range(H):
            j = H + h // (H // Hkv)
            w = s["rows"][a:b, h].double() @ s["rows"][a:b, j].double().t().contiguous() / math.sqrt(c["dh"])
            w[later] = -math.inf
            o[a:b, h] = torch.softmax(w, -1) @ s["rows"][a:b, j + Hkv].double()
    return o


def _round_e4m3(x):
    """To 4 significant bits and no finer than 2^-9, ties to even."""
    ulp = torch.exp2((torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6) * (1 + 1e-12))) - 3))
    return torch.round(x / ulp) * ulp


def _exponent(x):
    """The smallest e with max |x| <= 448 2^e over tokens and dims of x [n, Hkv, dh]; -118 at least."""
    top = x.abs().amax((0, 2)).clamp_min(2.0 ** -110)
    return torch.ceil(torch.log2(top / 448) - 1e-12).clamp_min(-118)


def _exact_cache(parts):
    """The values of one sequence's rows in the cache, stored in these calls one behind the other."""
    out = torch.cat(parts).double()
    cut = parts[0].shape[0]
    for a in range(0, out.shape[0], BLOCK):
        rows = out[a:a + BLOCK]
        n = min(max(cut - a, 0), rows.shape[0])
        e = _exponent(rows[:n]) if n else None
        if n:
            unit = torch.exp2(e)[:, None]
            rows[:n] = _round_e4m3(rows[:n] / unit) * unit
        if n < rows.shape[0]:
            more = _exponent(rows[n:])
            unit = torch.exp2(more if e is None else torch.maximum(e, more))[:, None]
            rows[:] = _round_e4m3(rows / unit) * unit
    return out


def _exact_kv8(c, s):
    ahead, out = _ahead(c), []
    for old, new in ((s["k0"], s["k"]), (s["v0"], s["v"])):
        y = torch.zeros((c["B"], c["L"] + ahead, c["Hkv"], c["dh"]), dtype=torch.float64, device="cuda")
        for b, (n0, n) in enumerate(zip(_starts(c), _counts(c))):
            y[b, :ahead + n] = _exact_cache([old[b, :n0], new[b, :n]])[n0 - ahead:]
        out.append(y)
    return tuple(out)


def _exact_att(c, s):
    G, Lq = c["H"] // c["Hkv"], c["Lq"]
    o = torch.zeros((c["B"], Lq, c["H"], c["dh"]), dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lens(c)):
        lo = max(0, n - c["window"] - Lq + 1) if c["window"] else 0
        keep = [j for j in range(min(c["sinks"], lo))] + list(range(lo, n))
        at = torch.tensor(keep, device="cuda")
        k, v = (_exact_cache([x[b, :n]])[at] for x in (s["k"], s["v"]))
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
    return {"norm": _exact_norm, "gemm": _exact_gemm, "pack": _exact_pack, "kv8": _exact_kv8, "att": _exact_att}[case["op"]](case, s)
