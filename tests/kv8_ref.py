"""The 8-bit cache and attention over it in float64, and helpers for its tests."""
import numpy as np

BLOCK, LEAST = 32, -118


def normal(key, shape, std=1.0):
    seed = [ord(c) for c in str(key)]
    return bf16(np.random.default_rng(seed).standard_normal(shape) * std)


def bf16(x):
    """To the nearest bf16, ties to even; as float32."""
    u = np.ascontiguousarray(np.asarray(x, np.float32)).view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(x), r, np.asarray(x, np.float32))


def to_dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def from_dev(t):
    return t.float().cpu().numpy()


def code(x):
    """To the nearest number of 4 significant bits and a multiple of 2^-9 (|x| <= 448), ties to even."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(np.where(np.isfinite(x) & (x != 0), x, 1.0))
    ulp = np.exp2(np.maximum(e - 4, -9).astype(np.float64))
    return np.rint(x / ulp) * ulp


def exponent(x):
    """The least e >= -118 for which every finite |x| is at most 448 2^e; over all but the second-last axis' head."""
    a = np.where(np.isfinite(x), np.abs(np.asarray(x, np.float64)), 0).max((0, 2))
    m, e = np.frexp(a)
    return np.maximum(np.where(a > 0, e - 9 + (m > 0.875), LEAST), LEAST)


class Cache:
    """Keys (or values) of one sequence: codes [L_cap][Hkv][dh] and exponents [L_cap / 32][Hkv]."""

    def __init__(self, L_cap, Hkv, dh):
        self.c = np.zeros((L_cap, Hkv, dh))
        self.e = np.full((L_cap // BLOCK, Hkv), LEAST)

    def store(self, x, start, count=None):
        n = len(x) if count is None else min(max(count, 0), len(x))
        first, last = max(start, 0), min(start + n, len(self.c))
        for blk in range(first // BLOCK, (last + BLOCK - 1) // BLOCK):
            lo, hi = max(first, blk * BLOCK), min(last, (blk + 1) * BLOCK)
            if lo >= hi:
                continue
            with np.errstate(all="ignore"):
                rows = np.asarray(x[lo - start:hi - start], np.float64)
            e = exponent(rows)
            here = self.c[blk * BLOCK:(blk + 1) * BLOCK]
            if lo == blk * BLOCK:
                here[:] = 0
            else:
                e = np.maximum(e, self.e[blk])
                here[:] = code(here * np.exp2((self.e[blk] - e).astype(np.float64))[:, None])
            self.e[blk] = e
            unit = np.exp2(e.astype(np.float64))[:, None]
            self.c[lo:hi] = np.where(np.isfinite(rows), code(np.where(np.isfinite(rows), rows, 0) / unit), np.nan)

    def values(self):
        return self.c * np.exp2(np.repeat(self.e, BLOCK, 0).astype(np.float64))[..., None]


def attention(q, k, v, n, window=0, sinks=0):
    """q [Lq][H][dh], k, v [n..][Hkv][dh] as the cache has them, n tokens: (o, bound on |computed - o|), by the
    kernel's roundings: weights in fp16 (2^-11 each), scores from fp32 sums of dh exact products,
    fp32 sums over n keys, a bf16 result (2^-8)."""
    Lq, H, dh = q.shape
    G = H // k.shape[1]
    o, tol = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(Lq):
        p = n - Lq + i
        j = np.arange(0, max(p + 1, 0))
        if window:
            j = j[(j > p - window) | (j < sinks)]
        if p < 0 or not len(j):
            continue
        for h in range(H):
            kk, vv = k[j, h // G], v[j, h // G]
            with np.errstate(all="ignore"):
                s = kk @ q[i, h].astype(np.float64) / np.sqrt(dh)
                off = ((np.abs(kk) @ np.abs(q[i, h].astype(np.float64))) / np.sqrt(dh) * (dh + 4)).max() * 2.0 ** -24
                w = np.exp(s - s.max())
                w /= w.sum()
                o[i, h] = w @ vv
                size = w @ np.abs(vv)
            rel = 2.0 ** -11 + 2 * off + (len(j) + 64) * 2.0 ** -24
            tol[i, h] = size * rel + np.abs(o[i, h]) * 2.0 ** -8 + 1e-37
    return o, tol
