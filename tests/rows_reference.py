"""Plain 64-bit numpy forms of the operators whose rows choose their own weights, for the tests."""
import numpy as np


def group_rows(ids, count):
    """(order, offsets): rows by group, ascending in each, those of no group last."""
    flat = np.asarray(ids).reshape(-1).astype(np.int64)
    key = np.where((flat < 0) | (flat >= count), count, flat)
    order = np.argsort(key, kind="stable").astype(np.int32)
    sizes = np.bincount(key, minlength=count + 1)[:count]
    return order, np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)


def route(logits, k, score, bias=None, groups=1, top_groups=1, group_top=1, renormalise=True, scale=1.0):
    """(experts [M,k], weights [M,k] in 64 bits); -inf and NaN logits are not there, +inf is the largest fp32."""
    M, E = logits.shape
    l64 = np.minimum(logits.astype(np.float64), float(np.finfo(np.float32).max))
    experts, weights = np.full((M, k), -1, np.int32), np.zeros((M, k))
    size = E // groups
    for m in range(M):
        l = l64[m]
        there = [e for e in range(E) if l[e] > -np.inf]
        if not there:
            continue
        s = np.zeros(E)
        with np.errstate(over="ignore"):
            if score == "softmax":
                s[there] = np.exp(l[there] - l[there].max())
                s /= s.sum()
            else:
                s[there] = 1.0 / (1.0 + np.exp(-l[there]))
        c = s + (0.0 if bias is None else bias.astype(np.float64))
        # a score grows with its logit: without a bias the logits themselves decide
        by = (lambda e: l[e]) if bias is None else (lambda e: c[e])
        if top_groups < groups:
            worth = {}
            for g in range(groups):
                mine = sorted((e for e in there if e // size == g), key=lambda e: (-by(e), e))[:group_top]
                if mine:
                    worth[g] = by(mine[0]) if group_top == 1 else sum(c[e] for e in mine)
            kept = sorted(worth, key=lambda g: (-worth[g], g))[:top_groups]
            there = [e for e in there if e // size in kept]
            if group_top == 2:
                by = lambda e: c[e]
        chosen = sorted(there, key=lambda e: (-by(e), e))[:k]
        w = s[chosen]
        if renormalise and chosen:
            # sigmoids far below 0 are e^l, whose ratios remain where the scores themselves underflow
            top = l[chosen].max()
            if top < -700.0:
                w = np.exp(l[chosen] - top)
            w = w / w.sum()
        experts[m, :len(chosen)], weights[m, :len(chosen)] = chosen, w * scale
    return experts, weights


def expert_rows(codes, sw, xq, sx, order, offsets, k, group):
    """(y, slack) [rows with an expert, N] in 64 bits and what fp32 sums over groups may be off by."""
    E, N, K = codes.shape
    total = int(offsets[-1])
    y, slack = np.zeros((total, N)), np.zeros((total, N))
    for e in range(E):
        r0, r1 = int(offsets[e]), int(offsets[e + 1])
        at = order[r0:r1] // k if k else np.arange(r0, r1)
        x, s = xq[at].astype(np.int64), sx[at].astype(np.float64)[:, None]
        w = codes[e].astype(np.int64)
        if group == 0:
            y[r0:r1] = (x @ w.T).astype(np.float64) * (s * sw[e].astype(np.float64)[None, :])
        else:
            G = K // 128
            acc = np.einsum("mgk,ngk->mng", x.reshape(-1, G, 128), w.reshape(N, G, 128)).astype(np.float64)
            terms = acc * sw[e].astype(np.float64)[None]
            y[r0:r1] = terms.sum(2) * s
            slack[r0:r1] = np.abs(terms).sum(2) * s * G * 2.0**-23
    return y, slack


def combine(y, experts, weights, add=None):
    """(out, bound): 64 bits, and what a sum in fp32 and one rounding to fp16 may be off by."""
    M, k = experts.shape
    rows = np.where((experts >= 0)[:, :, None], y.reshape(M, k, -1).astype(np.float64), 0.0)
    terms = rows * weights.astype(np.float64)[:, :, None]
    out, size = terms.sum(1), np.abs(terms).sum(1)
    if add is not None:
        out, size = out + add.astype(np.float64), size + np.abs(add.astype(np.float64))
    return out, (k + 1) * 2.0**-24 * size + 2.0**-11 * np.abs(out) + 2.0**-25


def adapters(a, b, scale, x, ids, y):
    """(out, bound).  The bound: each of the K products' additions is off by 2^-23 of the running sum of magnitudes at
    most (16 partial sums, then the splits, all in fp32: fewer than K additions one after the other); h is split to
    2^-22 of itself or 2^-37 of its row's largest; then R additions in fp32, the product with the scale and the final
    sum 2^-24 each, and half a step of fp16."""
    out = y.astype(np.float64)
    bound = np.zeros_like(out)
    R = a.shape[1]
    for m in range(x.shape[0]):
        l = int(ids[m])
        if not 0 <= l < a.shape[0]:
            continue
        al, bl, xm = a[l].astype(np.float64), b[l].astype(np.float64), x[m].astype(np.float64)
        h = al @ xm
        h_off = x.shape[1] * 2.0**-23 * (np.abs(al) @ np.abs(xm)) + 2.0**-22 * np.abs(h) + 2.0**-37 * np.abs(h).max()
        s = float(scale[l])
        out[m] += s * (bl @ h)
        bound[m] = abs(s) * (np.abs(bl) @ h_off + 2 * R * 2.0**-23 * (np.abs(bl) @ np.abs(h)))
    return out, bound + 2.0**-23 * np.abs(out) + 2.0**-11 * np.abs(out) + 2.0**-25
