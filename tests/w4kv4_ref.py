"""Plain numpy float64 definitions of the 4-bit operators, for their tests."""
import numpy as np

import synth


def bf16(x):
    """x rounded to bfloat16, as float64 (through float32, as a kernel's result is)."""
    with np.errstate(over="ignore"):
        f = np.asarray(x, np.float64).astype(np.float32)
    u = np.ascontiguousarray(f).view(np.uint32).astype(np.uint64)
    r = (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32)
    return np.where(np.isfinite(f), r.view(np.float32).astype(np.float64), f.astype(np.float64)).reshape(f.shape)


def quantise(x):
    """(codes, s, m) of x[..., dh] (bf16 values, float64) in groups of 32 dims."""
    g = x.reshape(x.shape[:-1] + (-1, 32))
    lo, hi = g.min(-1, keepdims=True), g.max(-1, keepdims=True)
    bad = ~np.isfinite(g).all(-1, keepdims=True)
    with np.errstate(all="ignore"):
        d = (hi - lo).astype(np.float32)  # the step is a product in fp32, so that ties fall as the kernel's
        s = bf16(np.where(np.isfinite(d), (d * np.float32(1 / 15)).astype(np.float64), (hi - lo) / 15))
        s = np.where(hi - lo < 2.0 ** -99, 0.0, s)
        c = np.where(s > 0, np.minimum(np.rint((g - lo) / np.where(s > 0, s, 1)), 15), 0)
    c, s, lo = np.where(bad, 0, c), np.where(bad, np.nan, s), np.where(bad, np.nan, lo)
    return c, s, lo


def cached(x):
    """What rows x[..., dh] stand for in the cache (float64, not rounded)."""
    c, s, m = quantise(x)
    return (m + s * c).reshape(x.shape)


def w4_weights(codes, scales, zeros, group):
    """W[N][K] in float64."""
    k = np.arange(codes.shape[1]) // group
    z = 8.0 if zeros is None else zeros[:, k]
    return scales[:, k] * (codes - z)


def visible(pos, n, window, sinks):
    """Whether the query at position pos sees each of n cached keys."""
    j = np.arange(n)
    see = j <= pos
    if window > 0:
        see &= (j > pos - window) | (j < sinks)
    return see


def attention(q, k, v, length, window, sinks):
    """o[Lq][H][dh] and sum_j p_j |v_j| of one sequence: q[Lq][H][dh], k, v
    [n][Hkv][dh], the last Lq of `length` tokens."""
    Lq, H, dh = q.shape
    Hkv = k.shape[1]
    o, mag = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(Lq):
        see = visible(length - Lq + i, length, window, sinks)
        if not see.any():
            continue
        for h in range(H):
            kv = h // (H // Hkv)
            w = k[:length][see, kv] @ q[i, h] / np.sqrt(dh)
            p = np.exp(w - w.max())
            p /= p.sum()
            o[i, h] = p @ v[:length][see, kv]
            mag[i, h] = p @ np.abs(v[:length][see, kv])
    return o, mag


def head_norm_rope(x, gain, eps, cos, sin):
    """x[..., heads, dh] with cos, sin[..., dh/2] of its token (None: not turned)."""
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    if cos is None:
        return x
    a, b = np.split(x, 2, -1)
    c, s = cos[..., None, :], sin[..., None, :]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def normal(tag, shape, std=1.0):
    """Seeded bf16 values as float64."""
    return synth.as_f32(synth.normal_bf16(synth.seed_of(*tag), shape, std=std)).astype(np.float64)


def to_dev(x, dtype="bf16"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32))
    return t.to(torch.bfloat16).cuda() if dtype == "bf16" else t.cuda()


def from_dev(t):
    return t.float().cpu().numpy().astype(np.float64)
