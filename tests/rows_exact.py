"""Adapters whose answer is exact: small whole numbers everywhere, so that every sum in fp32 is exact in any order and one
rounding, the last, is left; the projection all but cancels the adapter's term, so that this rounding hides nothing of it."""
import numpy as np


def draw(seed, M, L, K, N, R):
    """dict of a, b, scale, x, y, ids as for fq.adapters / group_rows, and `want`, fp16."""
    rng = np.random.default_rng([M, L, K, N, R, seed])
    # K a x of at most 2^23, two parts in bits to x
    room = int(2**23 // K)
    a_most = max(1, min(500, int(room ** (1 / 3))))
    x_most = max(1, min(1000, room // a_most))
    a = rng.integers(-a_most, a_most + 1, (L, R, K)).astype(np.float16)
    x = rng.integers(-x_most, x_most + 1, (M, K)).astype(np.float16)
    # three ranks a column: the sum over ranks is exact as well
    b = np.zeros((L, N, R), np.float16)
    at = rng.integers(0, R, (L, N, 3))
    np.put_along_axis(b, at, rng.choice([-2.0, -1.0, 1.0, 2.0], (L, N, 3)).astype(np.float16), 2)
    scale = (rng.choice([-1.0, 1.0], L) * 2.0 ** rng.integers(-12, -9, L)).astype(np.float32)
    ids = rng.integers(-1, L, M).astype(np.int32)
    ids[0] = L - 1
    case = dict(a=a, b=b, scale=scale, x=x, ids=ids)
    h = intermediate(case)
    for l in range(L):
        mine = np.abs(h[ids == l]) @ np.abs(b[l].astype(np.float64)).T
        assert mine.size == 0 or mine.max() < 2**24, "the sums over ranks would not be exact"
    y = (-term(case, h)).astype(np.float16)
    y[ids < 0] = rng.standard_normal((int((ids < 0).sum()), N)).astype(np.float16)
    case["y"] = y
    case["want"] = result(case, h)
    return case


def intermediate(case, steps=None):
    """A x by row in 64 bits, exact; steps: of the first so many 64 k only."""
    upto = case["x"].shape[1] if steps is None else 64 * steps
    h = np.zeros((case["x"].shape[0], case["a"].shape[1]))
    for l in range(case["a"].shape[0]):
        mine = case["ids"] == l
        h[mine] = case["x"][mine, :upto].astype(np.float64) @ case["a"][l, :, :upto].astype(np.float64).T
    return h


def halved(h):
    """h in the fp16 that a row's largest value leaves the others, without the rest."""
    top = np.abs(h).max(1, keepdims=True)
    power = 2.0 ** (14 - np.frexp(np.where(top > 0, top, 1.0))[1])
    return (h * power).astype(np.float16).astype(np.float64) / power


def term(case, h):
    out = np.zeros((h.shape[0], case["b"].shape[1]))
    for l in range(case["a"].shape[0]):
        mine = case["ids"] == l
        out[mine] = float(case["scale"][l]) * (h[mine] @ case["b"][l].astype(np.float64).T)
    return out


def result(case, h):
    return (case["y"].astype(np.float64) + term(case, h)).astype(np.float16)
