"""Plain forms of the rotation of heads, causal attention and the 8-bit cache in numpy, 64 bits, with bounds of how far the
kernels may be off, derived from what they round."""
import numpy as np

BLOCK = 16
HALF = 2.0**-11                 # half a step of fp16, relative
F32 = 2.0**-24                  # of fp32


def rotate(x, heads, kv, D, positions, freq, gamma_q=None, gamma_k=None, eps=1e-5, interleaved=False):
    """-> values in 64 bits and how far fp16 ones may be off."""
    M, rot = x.shape[0], 2 * len(freq)
    h = x[:, :(heads + kv) * D].astype(np.float64).reshape(M, heads + kv, D)
    for g, part in ((gamma_q, slice(0, heads)), (gamma_k, slice(heads, heads + kv))):
        if g is not None:
            p = h[:, part]
            h[:, part] = p / np.sqrt((p * p).mean(2, keepdims=True) + eps) * g.astype(np.float64)
    t = positions.astype(np.float64)[:, None] * freq.astype(np.float64)
    c, s = np.cos(t)[:, None], np.sin(t)[:, None]
    y, size = h.copy(), np.abs(h)
    at = np.arange(rot).reshape(rot // 2, 2).T if interleaved else np.arange(rot).reshape(2, rot // 2)
    a, b = h[..., at[0]], h[..., at[1]]
    y[..., at[0]], y[..., at[1]] = a * c - b * s, b * c + a * s
    size[..., at[0]] = size[..., at[1]] = np.abs(a) + np.abs(b)
    # fp32: the norm's sum and root (D additions of squares, half of their relative error in the root), two products, the
    # angle (2^-24 of an eighth of a turn and 2^-28 of the series) and the sums: 24 steps are more than all of it
    off = HALF * np.abs(y) + (D / 2 + 24) * F32 * size + 2.0**-25
    return y.reshape(M, -1), off.reshape(M, -1)


def attend(q, k, v, first, scale):
    """Causal attention of one head in 64 bits: query i of q [n, D] is token first + i and sees keys up to itself.
    -> values and how far fp16 ones may be off.  Rows that see nothing are zero."""
    n, D = q.shape
    L = k.shape[0]
    q, k, v = (z.astype(np.float64) for z in (q, k, v))
    if L == 0:
        return np.zeros((n, D)), np.zeros((n, D))
    score = scale * (q @ k.T)
    seen = np.arange(L)[None, :] <= first + np.arange(n)[:, None]
    score = np.where(seen, score, -np.inf)
    top = score.max(1, keepdims=True)
    p = np.where(seen, np.exp(score - np.where(np.isfinite(top), top, 0.0)), 0.0)
    total = p.sum(1, keepdims=True)
    total = np.where(total > 0, total, 1.0)
    y, size = p @ v / total, p @ np.abs(v) / total
    # a score: D products added in fp32 (a step each, two for the unit's alignment), scaled and rounded, and the exponent;
    # it is an error of the exponential's argument, of p and, averaged, of the sum
    largest = np.abs(np.where(seen, score, 0.0)).max(1, keepdims=True)
    s_off = (2 * D + 8) * F32 * scale * (np.abs(q) @ np.abs(k).T).max(1, keepdims=True) + 8 * F32 * (largest + 1)
    # p rounded to fp16 (half a step, and for the smallest of them 2^-34 of the largest), sums of L in fp32
    off = HALF * np.abs(y) + size * (HALF + 2 * s_off + (2 * L + 16) * F32) + L * 2.0**-34 * np.abs(v).max() + 2.0**-25
    return y, np.where(seen.any(1, keepdims=True), off, 0.0)


def grouped(q, k, v, heads, kv, first, scale):
    """attend for grouped heads: rows q [n, heads * D], k and v [L, kv * D]."""
    D, group = q.shape[1] // heads, heads // kv
    part = lambda z, h: z[:, h * D:(h + 1) * D]
    each = [attend(part(q, h), part(k, h // group), part(v, h // group), first, scale) for h in range(heads)]
    return np.concatenate([e[0] for e in each], 1), np.concatenate([e[1] for e in each], 1)


def stored(rows, kv):
    """What the cache stands for, of a sequence's fp16 rows [L, kv * D], in 64 bits: full blocks as code times scale."""
    L, width = rows.shape
    out = rows.astype(np.float64)
    for b in range(L // BLOCK):
        x = rows[b * BLOCK:(b + 1) * BLOCK].astype(np.float32).reshape(BLOCK, kv, -1)
        scale = (np.abs(x).max((0, 2)) / np.float32(127)).astype(np.float16)
        scale[scale == 0] = 1
        s = scale.astype(np.float32)[None, :, None]
        codes = np.clip(np.rint(x / s), -128, 127)
        out[b * BLOCK:(b + 1) * BLOCK] = (codes.astype(np.float64) * s).reshape(BLOCK, width)
    return out


def stored_half(rows, kv):
    """The same as reads give it: fp16, 65504 at most."""
    return np.clip(stored(rows, kv), -65504, 65504).astype(np.float16)
