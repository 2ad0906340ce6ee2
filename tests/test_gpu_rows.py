"""Rows that choose their own weights, on the GPU: grouping, routing to experts, the experts' linear layers and weighted
sums, low-rank adapters, and a run of them together, against plain forms in 64 bits (rows_reference)."""
import numpy as np
import pytest
import torch

import paper_2508_04405_amd as fq
from paper_2508_04405_amd import dev
import rows_reference as ref
from gpu_helpers import assert_y_close, say, to_dev

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = float("inf")


def host(t):
    return t.cpu().numpy()


# ---- grouping --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("count", [1, 2, 63, 64, 65, 256, 512])
@pytest.mark.parametrize("rows", [1, 2, 63, 65, 1023, 1024, 1025, 5000, 140001])
def test_group_rows(rows, count):
    say(f"group_rows rows={rows} count={count}")
    rng = np.random.default_rng([rows, count])
    ids = rng.integers(-1, count, rows).astype(np.int32)
    ids[rng.random(rows) < 0.02] = np.int32(2**31 - 1)       # of no group, like every id outside
    ids[rng.random(rows) < 0.02] = count
    ids[rng.random(rows) < 0.02] = np.int32(-2**31)
    order, offsets = fq.group_rows(to_dev(ids), count)
    want = ref.group_rows(ids, count)
    assert np.array_equal(host(offsets), want[1])
    assert np.array_equal(host(order), want[0])


@pytest.mark.parametrize("fill", [-1, 0, 6])
def test_group_rows_of_one_id(fill):
    for rows in (7, 3000):
        ids = np.full(rows, fill, np.int32)
        order, offsets = fq.group_rows(to_dev(ids), 7)
        want = ref.group_rows(ids, 7)
        assert np.array_equal(host(order), want[0]) and np.array_equal(host(offsets), want[1])


# ---- routing ---------------------------------------------------------------------------------------------------

def check_route(logits, k, bias=None, weight_bits=19, **kw):
    r = fq.route_experts(to_dev(logits), k, bias=None if bias is None else to_dev(bias), **kw)
    experts, weights = ref.route(logits, k, bias=bias, **kw)
    assert np.array_equal(host(r.experts), experts), np.argwhere(host(r.experts) != experts)[:5]
    got = host(r.weights).astype(np.float64)
    # fp32: an exponential good to 2^-22 whose argument, up to 32 away, is rounded to 2^-24 of itself, over a sum of such
    assert np.all(np.abs(got - weights) <= 2.0**-weight_bits * np.abs(weights) + 2.0**-140), np.abs(got - weights).max()
    order, offsets = ref.group_rows(experts, logits.shape[1])
    assert np.array_equal(host(r.order), order) and np.array_equal(host(r.offsets), offsets)
    return r


SHAPES = [(1, 8, 2), (1, 1, 1), (3, 2, 2), (17, 60, 4), (64, 64, 6), (65, 64, 6), (33, 160, 6), (130, 256, 8), (40, 512, 16),
          (2050, 72, 3), (70, 65, 5)]


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("M,E,k", SHAPES)
def test_route(M, E, k, score, renormalise):
    say(f"route M={M} E={E} k={k} {score} renormalise={renormalise}")
    rng = np.random.default_rng([M, E, k])
    logits = (2.0 * rng.standard_normal((M, E))).astype(np.float32)
    check_route(logits, k, score=score, renormalise=renormalise, scale=1.5)
    check_route(logits.astype(np.float16), k, score=score, renormalise=renormalise)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("M,E,k,groups,top_groups,group_top", [
    (5, 8, 2, 4, 2, 2), (33, 256, 8, 8, 4, 2), (9, 160, 6, 8, 3, 1), (66, 60, 4, 3, 1, 2), (7, 64, 6, 64, 10, 2),
    (20, 512, 16, 16, 16, 2), (12, 66, 5, 33, 7, 1), (1, 6, 3, 2, 1, 2)])
def test_route_groups_and_bias(M, E, k, groups, top_groups, group_top, score):
    say(f"route M={M} E={E} k={k} groups={groups}/{top_groups}/{group_top} {score}")
    rng = np.random.default_rng([M, E, groups])
    logits = (1.5 * rng.standard_normal((M, E))).astype(np.float32)
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32)
    for b in (bias, None):
        check_route(logits, k, bias=b, score=score, groups=groups, top_groups=top_groups, group_top=group_top)
        check_route(logits, k, bias=b, score=score, groups=groups, top_groups=top_groups, group_top=group_top, renormalise=False)


@pytest.mark.parametrize("M,E,k,groups,top_groups", [(40, 16, 3, 2, 1), (50, 100, 5, 4, 2), (70, 256, 8, 8, 4), (21, 510, 16, 17, 6)])
def test_route_of_fp16_logits_with_bias_and_groups(M, E, k, groups, top_groups):
    """Logits of 16 bits: scores that are equal without the bias are the rule."""
    say(f"route fp16 M={M} E={E} k={k} groups={groups}/{top_groups}")
    rng = np.random.default_rng([M, E, 16])
    logits = rng.standard_normal((M, E)).astype(np.float16)
    logits[:, ::3] = np.float16(0.5)
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32)
    bias[: E // 2] = 0.25
    for score in ("softmax", "sigmoid"):
        check_route(logits, k, bias=bias, score=score)
        check_route(logits, k, bias=bias, score=score, groups=groups, top_groups=top_groups, group_top=2)
        check_route(logits, k, score=score, groups=groups, top_groups=top_groups, group_top=2, renormalise=False)


@pytest.mark.parametrize("kw", [dict(score="softmax"), dict(score="sigmoid", renormalise=False),
                                dict(score="sigmoid", groups=8, top_groups=3, group_top=2),
                                dict(score="softmax", groups=8, top_groups=2, group_top=1)])
def test_route_ties_go_to_the_lowest_index(kw):
    rng = np.random.default_rng(3)
    logits = rng.integers(-1, 2, (50, 64)).astype(np.float32)
    logits[0] = 0.0
    logits[1, ::2] = -0.0                                     # one value with 0
    logits[1, 1::2] = 0.0
    check_route(logits, 6, **kw)
    check_route(logits, 6, bias=np.zeros(64, np.float32), **kw)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("kw", [dict(score="softmax"), dict(score="softmax", renormalise=False), dict(score="sigmoid"),
                                dict(score="sigmoid", groups=5, top_groups=2, group_top=2)])
def test_route_of_masked_experts(kw, bias):
    """Rows with nothing, one, or fewer than k experts, masks of -inf, of the types' lowest values and NaN, and +inf."""
    rng = np.random.default_rng(4)
    b = (0.1 * rng.standard_normal(40)).astype(np.float32) if bias else None
    for dtype in (np.float32, np.float16):
        logits = rng.standard_normal((80, 40)).astype(dtype)
        logits[0] = -INF
        logits[1] = np.nan
        logits[2] = -INF
        logits[2, 17] = -3.0
        logits[3] = -INF
        logits[3, [5, 39]] = 1.0
        logits[4, rng.random(40) < 0.5] = np.nan
        logits[5, rng.random(40) < 0.9] = -INF
        logits[6] = np.finfo(dtype).min                       # there, but as low as can be
        logits[7, :39] = np.finfo(dtype).min
        logits[8, 3] = INF
        logits[9, 8:32] = -INF
        # scores may underflow to 0 in 32 bits where they are not 0 in 64, hence the absolute part of the bound
        check_route(logits, 4, bias=b, **kw)


def test_route_of_scores_closer_than_fp32_tells():
    """Sigmoid scores of neighbouring logits near 1 differ by less than fp32 resolves; a bias decides between others."""
    logits = np.float32(12.0) + np.arange(64, dtype=np.float32)[None, ::-1] * np.float32(2.0**-20)
    logits = np.repeat(logits, 3, 0).copy()
    check_route(logits, 8, bias=np.zeros(64, np.float32), score="sigmoid")
    check_route(logits, 8, bias=np.full(64, 0.25, np.float32), score="sigmoid", renormalise=False)
    check_route(logits, 8, score="sigmoid", groups=4, top_groups=2, group_top=2)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("M,E,k", [(70, 8, 2), (33, 40, 15), (100, 256, 8), (20, 512, 16), (40, 64, 6), (9, 16, 16)])
def test_route_of_pairs_that_fp32_cannot_tell_apart(M, E, k, score):
    """Experts in pairs whose scores differ by less than fp32 scores are good to, in either order: few at a time (some
    rows), or all (others); the last chosen and the first left out among them."""
    rng = np.random.default_rng([M, E, k, 7])
    logits = (1.5 * rng.standard_normal((M, E))).astype(np.float32)
    for m in range(M):
        pairs = rng.permutation(E).reshape(-1, 2)[:rng.integers(1, E // 2 + 1)]
        up = rng.integers(0, 2, len(pairs)).astype(bool)
        logits[m, pairs[:, 1]] = np.nextafter(logits[m, pairs[:, 0]], np.where(up, np.inf, -np.inf).astype(np.float32))
    zero = np.zeros(E, np.float32)
    check_route(logits, k, bias=zero, score=score)
    check_route(logits, k, bias=zero, score=score, renormalise=False)
    if E % 8 == 0:                                            # groups that repeat each other, a little higher or lower
        size = E // 8
        logits[:, size:2 * size] = np.nextafter(logits[:, :size], np.float32(np.inf))
        logits[:, 5 * size:6 * size] = np.nextafter(logits[:, :size], np.float32(-np.inf))
        for top_groups in (1, 4):
            if k <= top_groups * size:
                check_route(logits, k, bias=zero, score=score, groups=8, top_groups=top_groups, group_top=2)
                check_route(logits, k, bias=zero, score=score, groups=8, top_groups=top_groups, group_top=1)


# ---- the experts' linear layers ----------------------------------------------------------------------------------

def draw_experts(rng, E, N, K, group):
    codes = np.clip(np.rint(9.0 * rng.standard_normal((E, N, K))), -32, 31).astype(np.int8)
    sw = (0.002 * (0.5 + rng.random((E, N) if group == 0 else (E, N, K // 128)))).astype(np.float16)
    return codes, sw


def draw_rows(rng, rows, K, bits):
    most = 31 if bits == 6 else 127
    xq = np.clip(np.rint(most / 4.0 * rng.standard_normal((rows, K))), -most - 1, most).astype(np.int8)
    return xq, ((0.5 + rng.random(rows)) / most).astype(np.float16)


def check_experts(rng, M, E, k, N, K, group, bits, experts, sorted_rows=False, scatter=False):
    codes, sw = draw_experts(rng, E, N, K, group)
    xq, sx = draw_rows(rng, M * k if sorted_rows else M, K, bits)
    packed = fq.pack_experts(to_dev(codes), to_dev(sw), group)
    order, offsets = ref.group_rows(experts, E)
    args = (packed, N, K, to_dev(xq), to_dev(sx), to_dev(order), to_dev(offsets))
    kw = dict(group=group, k=0 if sorted_rows else k, scatter=scatter)
    total = int(offsets[-1])
    want, slack = ref.expert_rows(codes, sw, xq, sx, order, offsets, 0 if sorted_rows else k, group)
    rows = order[:total] if scatter else np.arange(total)
    rest = np.setdiff1d(np.arange(M * k), rows)
    for form in range(7):                                     # the library's choice, then every kernel
        out = torch.full((M * k, N), 7.0, dtype=torch.float16, device=DEV)
        if form == 0:
            fq.expert_linear(*args, out=out, **kw)
        else:
            dev.expert_linear(form, *args, out=out, **kw)
        got = host(out)
        if total:
            assert_y_close(got[rows], want.astype(np.float16), slack if group else None)
        assert np.all(got[rest] == 7.0), "rows without an expert are left as they were"


def some_experts(rng, M, E, k, dropped=0.0):
    ids = np.stack([rng.permutation(E)[:k] for _ in range(M)]).astype(np.int32)
    ids[rng.random(M) < dropped] = -1
    return ids


@pytest.mark.parametrize("group,bits", [(0, 6), (0, 8), (128, 8), (128, 6)])
@pytest.mark.parametrize("M,E,k,N,K,sorted_rows,scatter,dropped", [
    (1, 4, 1, 32, 128, False, False, 0.0), (1, 8, 2, 96, 256, False, True, 0.0), (3, 5, 3, 160, 384, True, True, 0.0),
    (7, 70, 2, 64, 128, False, False, 0.3), (40, 4, 2, 288, 640, False, False, 0.1), (70, 3, 1, 128, 1152, True, False, 0.2),
    (150, 6, 4, 544, 256, False, True, 0.1), (300, 3, 2, 320, 512, True, True, 0.0), (600, 2, 1, 1056, 384, False, False, 0.05),
    (33, 12, 5, 4128, 128, False, False, 0.1), (2, 3, 2, 64, 9088, False, True, 0.0)])
def test_expert_linear(M, E, k, N, K, sorted_rows, scatter, dropped, group, bits):
    say(f"experts M={M} E={E} k={k} N={N} K={K} sorted={sorted_rows} scatter={scatter} group={group} bits={bits}")
    rng = np.random.default_rng([M, E, N, K, group])
    check_experts(rng, M, E, k, N, K, group, bits, some_experts(rng, M, E, k, dropped), sorted_rows, scatter)


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("sizes", [[0, 0, 0], [1, 0, 0], [0, 0, 1], [200, 0, 1], [0, 129, 0], [31, 32, 33], [127, 128, 129],
                                   [63, 64, 65], [257, 1, 255], [16, 17, 15]])
def test_expert_linear_group_sizes(sizes, group):
    """Experts with no rows, with one, and with rows on either side of the kernels' row tiles."""
    say(f"experts of sizes {sizes} group={group}")
    rng = np.random.default_rng(sizes + [group])
    ids = np.concatenate([np.full(n, e, np.int32) for e, n in enumerate(sizes)] + [np.full(3, -1, np.int32)])
    rng.shuffle(ids)
    for sorted_rows in (False, True):
        check_experts(rng, ids.size, 3, 1, 288, 384, group, 8, ids[:, None], sorted_rows, not sorted_rows)


def test_expert_linear_same_expert_in_several_slots():
    rng = np.random.default_rng(9)
    ids = rng.integers(0, 3, (50, 4)).astype(np.int32)        # a token may name an expert twice
    check_experts(rng, 50, 3, 4, 96, 256, 0, 8, ids)


def test_expert_linear_equals_the_dense_layer():
    """All rows with one expert: the rows of the dense call on that expert's weights, to the last place."""
    rng = np.random.default_rng(10)
    for M, N, K in ((5, 256, 1024), (200, 544, 640)):
        codes, sw = draw_experts(rng, 2, N, K, 0)
        xq, sx = (to_dev(v) for v in draw_rows(rng, M, K, 8))
        packed = fq.pack_experts(to_dev(codes), to_dev(sw))
        order, offsets = fq.group_rows(torch.ones((M,), dtype=torch.int32, device=DEV), 2)
        y = fq.expert_linear(packed, N, K, xq, sx, order, offsets, k=1)
        dense = fq.gemm_w6a8(packed[1], N, K, xq=xq, sx=sx)
        assert_y_close(host(y), host(dense))


@pytest.mark.parametrize("with_add", [False, True])
@pytest.mark.parametrize("M,k,N", [(1, 1, 32), (3, 6, 96), (257, 2, 4096), (5, 16, 5248)])
def test_combine(M, k, N, with_add):
    say(f"combine M={M} k={k} N={N} add={with_add}")
    rng = np.random.default_rng([M, k, N])
    y = rng.standard_normal((M * k, N)).astype(np.float16)
    experts = rng.integers(-1, 5, (M, k)).astype(np.int32)
    y[experts.reshape(-1) < 0] = np.nan                       # rows that were never written
    weights = rng.random((M, k)).astype(np.float32)
    add = rng.standard_normal((M, N)).astype(np.float16) if with_add else None
    want, bound = ref.combine(y, experts, weights, add)
    d_add = to_dev(add) if with_add else None
    out = fq.combine_experts(to_dev(y), to_dev(experts), to_dev(weights), add=d_add)
    assert np.all(np.abs(host(out).astype(np.float64) - want) <= bound)
    if with_add:                                              # in place
        same = fq.combine_experts(to_dev(y), to_dev(experts), to_dev(weights), add=d_add, out=d_add)
        assert torch.equal(same, out)


# ---- adapters ----------------------------------------------------------------------------------------------------

def draw_adapters(rng, L, R, K, N):
    a = (rng.standard_normal((L, R, K)) / np.sqrt(K)).astype(np.float16)
    b = (0.1 * rng.standard_normal((L, N, R))).astype(np.float16)
    return a, b, (0.5 + rng.random(L)).astype(np.float32)


def check_adapters(a, b, scale, x, ids, y, in_place=False):
    d = [to_dev(v) for v in (a, b, scale, x)]
    order, offsets = fq.group_rows(to_dev(ids), a.shape[0])
    dy = to_dev(y)
    out = fq.adapters(*d, order, offsets, dy, out=dy if in_place else None)
    want, bound = ref.adapters(a, b, scale, x, ids, y)
    got = host(out).astype(np.float64)
    assert np.all(np.abs(got - want) <= bound), (np.abs(got - want) / bound).max()
    none = (ids < 0) | (ids >= a.shape[0])
    assert np.array_equal(host(out)[none], y[none])
    return out


@pytest.mark.parametrize("R", [16, 32, 48, 64, 80, 128, 144, 256])
@pytest.mark.parametrize("M,L,K,N", [(1, 1, 128, 32), (2, 3, 256, 96), (17, 2, 640, 160), (40, 30, 1152, 544), (150, 4, 384, 1056)])
def test_adapters(M, L, K, N, R):
    say(f"adapters M={M} L={L} K={K} N={N} R={R}")
    rng = np.random.default_rng([M, L, K, N, R])
    a, b, scale = draw_adapters(rng, L, R, K, N)
    x, y = rng.standard_normal((M, K)).astype(np.float16), rng.standard_normal((M, N)).astype(np.float16)
    ids = rng.integers(-1, L, M).astype(np.int32)
    ids[0] = L - 1
    one = check_adapters(a, b, scale, x, ids, y)
    two = check_adapters(a, b, scale, x, ids, y, in_place=True)
    assert torch.equal(one, two)


@pytest.mark.parametrize("sizes", [[0, 0], [1, 0], [0, 1], [15, 16, 17], [33, 0, 64], [0, 300, 0]])
def test_adapters_group_sizes(sizes):
    rng = np.random.default_rng(sizes)
    L, R, K, N = len(sizes), 16, 256, 352
    ids = np.concatenate([np.full(n, i, np.int32) for i, n in enumerate(sizes)] + [np.full(20, -1, np.int32)])
    rng.shuffle(ids)
    a, b, scale = draw_adapters(rng, L, R, K, N)
    M = ids.size
    check_adapters(a, b, scale, rng.standard_normal((M, K)).astype(np.float16), ids, rng.standard_normal((M, N)).astype(np.float16))


def test_adapters_of_a_long_row():
    """K that is split over workgroups, the deepest layer of the benchmark."""
    rng = np.random.default_rng(12)
    a, b, scale = draw_adapters(rng, 2, 32, 28672, 96)
    x = rng.standard_normal((5, 28672)).astype(np.float16)
    check_adapters(a, b, scale, x, np.array([0, 1, -1, 0, 1], np.int32), rng.standard_normal((5, 96)).astype(np.float16))


@pytest.mark.parametrize("R", [16, 48, 64, 128])
def test_adapters_of_many_rows_and_a_long_row(R):
    """Pieces of 32 rows, K split over workgroups."""
    rng = np.random.default_rng([15, R])
    a, b, scale = draw_adapters(rng, 2, R, 8192, 96)
    ids = rng.integers(-1, 2, 100).astype(np.int32)
    check_adapters(a, b, scale, rng.standard_normal((100, 8192)).astype(np.float16), ids, rng.standard_normal((100, 96)).astype(np.float16))


@pytest.mark.parametrize("R,N", [(16, 20608), (32, 10304), (48, 6912), (64, 5152), (80, 4128), (112, 2976), (128, 2592)])
def test_adapters_in_pieces_of_32_rows(R, N):
    """So many rows that both launches take them 32 at a time."""
    rng = np.random.default_rng([16, R])
    a, b, scale = draw_adapters(rng, 2, R, 4096, N)
    ids = np.concatenate([np.zeros(37, np.int32), np.ones(1123, np.int32), np.full(40, -1, np.int32)])
    rng.shuffle(ids)
    check_adapters(a, b, scale, rng.standard_normal((1200, 4096)).astype(np.float16), ids, rng.standard_normal((1200, N)).astype(np.float16))


def test_adapters_keep_small_and_large_rows_apart():
    """The intermediate keeps 32 bits: rows whose A x lies outside fp16's range on either side, next to ordinary ones; a
    row that is not finite stays by itself."""
    rng = np.random.default_rng(13)
    L, R, K, N = 2, 16, 512, 64
    a, b, scale = draw_adapters(rng, L, R, K, N)
    a = (a.astype(np.float32) * 200).astype(np.float16)
    x = rng.standard_normal((16, K)).astype(np.float16)
    x[1] = (x[1].astype(np.float32) * 8000).astype(np.float16)        # A x up to 2e6
    x[2] = (x[2].astype(np.float32) * 2.0**-12).astype(np.float16)
    x[3] = 0.0
    a[:, 3:] = (a[:, 3:].astype(np.float32) * 2.0**-9).astype(np.float16)   # ranks far below the first three
    b = (b.astype(np.float32) * 1e-2).astype(np.float16)
    ids = np.tile(np.array([0, 1], np.int32), 8)
    y = rng.standard_normal((16, N)).astype(np.float16)
    out = check_adapters(a, b, scale, x, ids, y)
    x[4, 7] = np.inf
    x[5] = np.nan
    order, offsets = fq.group_rows(to_dev(ids), L)
    got = host(fq.adapters(*(to_dev(v) for v in (a, b, scale, x)), order, offsets, to_dev(y)))
    fine = [m for m in range(16) if m not in (4, 5)]
    assert np.array_equal(got[fine], host(out)[fine])


def test_adapters_of_lower_rank_padded_with_zeros():
    rng = np.random.default_rng(14)
    a, b, scale = draw_adapters(rng, 3, 32, 256, 96)
    a[1, 8:] = 0.0
    x, y = rng.standard_normal((9, 256)).astype(np.float16), rng.standard_normal((9, 96)).astype(np.float16)
    ids = np.arange(9, dtype=np.int32) % 3
    got = check_adapters(a, b, scale, x, ids, y)
    b[1, :, 8:] = 1000.0                                       # what zero rows of A meet does not matter
    assert torch.equal(got, check_adapters(a, b, scale, x, ids, y))


# ---- together ----------------------------------------------------------------------------------------------------

class FeedForward:
    """A batch through routed experts with adapters on the projection after them, as a program would run it."""

    def __init__(self, M, E, k, H, F, L, R, group, seed):
        rng = np.random.default_rng(seed)
        self.M, self.E, self.k, self.H, self.F, self.group = M, E, k, H, F, group
        up, down = draw_experts(rng, E, 2 * F, H, group), draw_experts(rng, E, H, F, group)
        proj = draw_experts(rng, 1, H, H, group)
        self.up, self.down = (fq.pack_experts(to_dev(c), to_dev(s), group) for c, s in (up, down))
        self.proj = fq.pack_experts(to_dev(proj[0]), to_dev(proj[1]), group)[0]
        self.lora = [to_dev(v) for v in draw_adapters(rng, L, R, H, H)]
        self.L = L
        self.gain = to_dev((1.0 + 0.1 * rng.standard_normal(H)).astype(np.float16))
        self.bias = to_dev((0.1 * rng.standard_normal(E)).astype(np.float32))
        self.ws = fq.make_workspace(M, H, H)
        self.x = to_dev(rng.standard_normal((M, H)).astype(np.float16))
        logits = (1.5 * rng.standard_normal((M, E))).astype(np.float32)
        if M > 2:
            logits[2] = -INF                                  # a padding token
        self.logits = to_dev(logits)
        self.ids = to_dev(rng.integers(-1, L, M).astype(np.int32))

    def run(self):
        s = {}
        s["route"] = r = fq.route_experts(self.logits, self.k, score="sigmoid", bias=self.bias, scale=1.5)
        s["xq"], s["sx"] = fq.rmsnorm_quant(self.x, self.gain, 1e-5, 8)
        s["gate_up"] = fq.expert_linear(self.up, 2 * self.F, self.H, s["xq"], s["sx"], r.order, r.offsets, group=self.group, k=self.k)
        s["hq"], s["hs"] = fq.swiglu_quant(s["gate_up"], 8)
        s["slots"] = fq.expert_linear(self.down, self.H, self.F, s["hq"], s["hs"], r.order, r.offsets, group=self.group, scatter=True)
        s["out"] = fq.combine_experts(s["slots"], r.experts, r.weights, add=self.x)
        s["order"], s["offsets"] = fq.group_rows(self.ids, self.L)
        s["y"] = fq.gemm_w6a8(self.proj, self.H, self.H, self.group, x_fp16=s["out"], workspace=self.ws)
        s["z"] = fq.adapters(*self.lora, s["out"], s["order"], s["offsets"], s["y"])
        return s


@pytest.mark.parametrize("M,E,k,H,F,group", [(1, 8, 2, 256, 128, 0), (5, 16, 4, 256, 384, 128), (90, 6, 2, 384, 256, 0)])
def test_feed_forward(M, E, k, H, F, group):
    """Each operator of the run against its plain form on the GPU's own inputs to it."""
    f = FeedForward(M, E, k, H, F, 3, 16, group, [M, E, H])
    s = f.run()
    r = s["route"]
    order, offsets = host(r.order), host(r.offsets)
    total = int(offsets[-1])
    experts, weights = ref.route(host(f.logits), k, "sigmoid", bias=host(f.bias), scale=1.5)
    assert np.array_equal(host(r.experts), experts)
    unpacked = [[fq.unpack_w6(w[e], n, kk, group) for e in range(E)] for w, n, kk in ((f.up, 2 * F, H), (f.down, H, F))]
    codes = [np.stack([host(c) for c, _ in layer]) for layer in unpacked]
    scales = [np.stack([host(v) for _, v in layer]) for layer in unpacked]
    want, slack = ref.expert_rows(codes[0], scales[0], host(s["xq"]), host(s["sx"]), order, offsets, k, group)
    assert_y_close(host(s["gate_up"])[:total], want.astype(np.float16), slack if group else None)
    want, slack = ref.expert_rows(codes[1], scales[1], host(s["hq"]), host(s["hs"]), order, offsets, 0, group)
    assert_y_close(host(s["slots"])[order[:total]], want.astype(np.float16), slack if group else None)
    want, bound = ref.combine(host(s["slots"]), experts, host(r.weights), host(f.x))
    assert np.all(np.abs(host(s["out"]).astype(np.float64) - want) <= bound)
    a, b, scale = (host(v) for v in f.lora)
    want, bound = ref.adapters(a, b, scale, host(s["out"]), host(f.ids), host(s["y"]))
    assert np.all(np.abs(host(s["z"]).astype(np.float64) - want) <= bound)


def test_feed_forward_captured_and_on_another_stream():
    """The run on a stream of its own, and captured into a graph that is replayed on new inputs between eager runs; rows
    of slots without an expert (their content is whatever the buffers held) are not compared."""
    f = FeedForward(33, 10, 3, 256, 256, 4, 32, 0, 21)
    eager = f.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = f.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for name in ("out", "y", "z"):
        assert torch.equal(eager[name], again[name]), name
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            kept = f.run()
    torch.cuda.synchronize()
    g = torch.Generator(device=DEV)
    for seed in range(4):
        g.manual_seed(seed)
        f.x.copy_(torch.randn(f.x.shape, generator=g, device=DEV))
        f.logits.copy_(torch.randn(f.logits.shape, generator=g, device=DEV))
        f.ids.copy_(torch.randint(-1, f.L, f.ids.shape, generator=g, device=DEV))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = f.run()
        torch.cuda.synchronize()
        for name in ("out", "y", "z"):
            assert torch.equal(eager[name], kept[name]), (seed, name)
        for i in range(4):
            assert torch.equal(eager["route"][i], kept["route"][i]), (seed, i)


# ---- limits and company ------------------------------------------------------------------------------------------

def test_rows_past_32_bits():
    """Outputs of more than 2^32 bytes: the last rows, through every kernel of the experts, the sum and the adapters."""
    rng = np.random.default_rng(30)
    E, N, K, slots = 2, 32768, 128, 70000
    codes, sw = draw_experts(rng, E, N, K, 0)
    xq, sx = draw_rows(rng, slots, K, 8)
    ids = (np.arange(slots) % 2).astype(np.int32)
    order, offsets = ref.group_rows(ids, E)
    args = (fq.pack_experts(to_dev(codes), to_dev(sw)), N, K, to_dev(xq), to_dev(sx), to_dev(order), to_dev(offsets))
    at = np.array([0, 34999, 35000, 65535, 65536, 69998, 69999])            # sorted rows
    want, _ = ref.expert_rows(codes, sw, xq[order[at]], sx[order[at]], np.arange(at.size), np.array([0, 2, at.size]), 1, 0)
    out = torch.empty((slots, N), dtype=torch.float16, device=DEV)
    for form in (2, 3, 4, 5, 6):
        say(f"form {form}")
        out.fill_(7.0)
        dev.expert_linear(form, *args, k=1, scatter=True, out=out)
        assert_y_close(host(out[torch.from_numpy(order[at]).long().to(DEV)]), want.astype(np.float16))
    M = slots // 2
    experts = torch.zeros((M, 2), dtype=torch.int32, device=DEV)
    weights = torch.rand((M, 2), dtype=torch.float32, device=DEV)
    sums = fq.combine_experts(out, experts, weights)
    rows = host(out[-6:])
    want, bound = ref.combine(rows, np.zeros((3, 2), np.int32), host(weights[-3:]))
    assert np.all(np.abs(host(sums[-3:]).astype(np.float64) - want) <= bound)
    del sums
    a, b, scale = draw_adapters(rng, 2, 16, K, N)
    x = rng.standard_normal((slots, K)).astype(np.float16)
    keep = host(out[-4:])
    fq.adapters(to_dev(a), to_dev(b), to_dev(scale), to_dev(x), to_dev(order), to_dev(offsets), out, out=out)
    want, bound = ref.adapters(a, b, scale, x[-4:], ids[-4:], keep)
    assert np.all(np.abs(host(out[-4:]).astype(np.float64) - want) <= bound)


def test_calls_on_two_streams_at_once():
    """Each call has a workspace of its own unless one is given: two streams' calls do not disturb each other."""
    rng = np.random.default_rng(31)
    runs = [FeedForward(90, 6, 2, 256, 256, 3, 16, 0, seed) for seed in (40, 41)]
    alone = [f.run() for f in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        both = []
        for f, st in zip(runs, streams):
            with torch.cuda.stream(st):
                both.append(f.run())
        torch.cuda.synchronize()
        for one, two in zip(alone, both):
            for name in ("out", "y", "z"):
                assert torch.equal(one[name], two[name]), name


def test_given_workspaces_and_refusals_on_the_device():
    ids = torch.randint(-1, 5, (3000,), dtype=torch.int32, device=DEV)
    ws = torch.full((1 << 20,), 255, dtype=torch.uint8, device=DEV)          # any content
    for got, want in zip(fq.group_rows(ids, 5, workspace=ws), fq.group_rows(ids, 5)):
        assert torch.equal(got, want)
    logits = torch.randn((100, 16), device=DEV)
    for got, want in zip(fq.route_experts(logits, 3, workspace=ws), fq.route_experts(logits, 3)):
        assert torch.equal(got, want)
    with pytest.raises(fq.FlexQError):
        fq.group_rows(ids, 5, workspace=ws[:64])
    with pytest.raises(fq.FlexQError):
        fq.group_rows(ids, 5, workspace=torch.zeros(1 << 20))                # not on the device
    with pytest.raises(fq.FlexQError):
        fq.group_rows(ids[::2], 5)
    with pytest.raises(fq.FlexQError):
        fq.route_experts(logits, 17)
    with pytest.raises(fq.FlexQError):
        fq.route_experts(logits, 3, groups=5)
    with pytest.raises(fq.FlexQError):
        fq.route_experts(logits, 3, bias=torch.zeros(15, device=DEV))
    assert fq.route_experts(logits, 3, group=False).order is None
