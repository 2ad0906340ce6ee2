"""Rows that choose their own weights, on the GPU, at the ends of their ranges: many groups, very many rows."""
import numpy as np
import pytest
import torch

import paper_2508_04405_amd as fq
import rows_exact
import rows_reference as ref
from gpu_helpers import say, to_dev
from test_gpu_rows import DEV, check_experts, check_route, draw_adapters, host, some_experts

pytestmark = pytest.mark.gpu


def grouped(ids, count):
    """(order, offsets) by torch, for more rows than the host sorts quickly."""
    key = torch.where((ids < 0) | (ids >= count), count, ids).long().reshape(-1)
    sizes = torch.bincount(key, minlength=count + 1)[:count]
    return torch.sort(key, stable=True)[1].int(), torch.cat([sizes.new_zeros(1), sizes.cumsum(0)]).int()


@pytest.mark.parametrize("rows,count,low", [(256 * 32768, 3, -1), (256 * 32768 + 1, 3, -1), (9000001, 512, -1), (10000000, 1, 0),
                                            (20000003, 257, -1)])
def test_more_rows_than_256_full_blocks(rows, count, low):
    """Blocks of 32768 rows, as many as their counts of 16 bits hold, all of one group among them."""
    say(f"group_rows rows={rows} count={count}")
    g = torch.Generator(device=DEV)
    g.manual_seed(rows)
    ids = torch.randint(low, count, (rows,), generator=g, device=DEV, dtype=torch.int32)
    ids[rows // 2:rows // 2 + 100000] = count - 1
    for got, want in zip(fq.group_rows(ids, count), grouped(ids, count)):
        assert torch.equal(got, want)


def test_routing_of_more_tokens_than_256_full_blocks():
    g = torch.Generator(device=DEV)
    g.manual_seed(70)
    M, E, k = 1200001, 9, 8
    logits = torch.randn((M, E), generator=g, device=DEV)
    logits[::1000] = -float("inf")
    r = fq.route_experts(logits, k)
    best = torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :k].int()
    best[::1000] = -1
    assert torch.equal(r.experts, best)
    for got, want in zip((r.order, r.offsets), grouped(r.experts, E)):
        assert torch.equal(got, want)
    at = torch.tensor([0, 1, 31, 32, M // 2, M - 2, M - 1], device=DEV)
    experts, weights = ref.route(host(logits[at]), k, "softmax")
    assert np.all(np.abs(host(r.weights[at]) - weights) <= 18 * 2.0**-24 * weights + 2.0**-146)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("M,E,k,groups,top_groups", [(40, 512, 16, 64, 2), (33, 512, 8, 64, 63), (70, 256, 8, 32, 5), (20, 448, 7, 64, 1),
                                                     (40, 512, 16, 2, 1)])
def test_routing_by_many_groups(M, E, k, groups, top_groups, score):
    say(f"route M={M} E={E} k={k} groups={groups}/{top_groups} {score}")
    rng = np.random.default_rng([M, E, groups, 71])
    logits = (1.5 * rng.standard_normal((M, E))).astype(np.float32)
    logits[:, rng.random(E) < 0.1] = -np.inf
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32)
    for b in (bias, None):
        for group_top in (1, 2):
            check_route(logits, k, bias=b, score=score, groups=groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("M,E,k,dropped", [(300, 512, 3, 0.1), (900, 65, 2, 0.0), (1, 512, 16, 0.0), (40, 128, 2, 0.5), (2000, 511, 2, 0.0)])
def test_many_experts(M, E, k, dropped, group):
    """Every kernel; experts beyond those that one look at the offsets sees."""
    say(f"experts M={M} E={E} k={k} group={group}")
    rng = np.random.default_rng([M, E, k, group, 72])
    ids = some_experts(rng, M, E, k, dropped)
    if M > 1:
        ids[0, 0] = E - 1
    check_experts(rng, M, E, k, 96, 256, group, 8, ids)
    check_experts(rng, M, E, k, 96, 256, group, 8, ids, sorted_rows=True, scatter=True)


@pytest.mark.parametrize("R", [16, 48, 64])
@pytest.mark.parametrize("L", [63, 64, 65, 128, 512])
def test_many_adapters(L, R):
    """Adapters, and the rows without one, beyond those that one look at the offsets sees; to the last bit."""
    say(f"adapters L={L} R={R}")
    for M in (3, 200, 700):
        case = rows_exact.draw(4, M, L, 256, 96, R)
        order, offsets = fq.group_rows(to_dev(case["ids"]), L)
        y = to_dev(case["y"])
        for out in (None, y):
            got = fq.adapters(*(to_dev(case[n]) for n in ("a", "b", "scale", "x")), order, offsets, y, out=out)
            assert np.array_equal(host(got), case["want"])


def test_the_most_rows_of_adapters():
    """2^24 rows, the last ones checked."""
    M, L, R, K, N = 1 << 24, 3, 16, 128, 32
    rng = np.random.default_rng(73)
    a, b, scale = draw_adapters(rng, L, R, K, N)
    g = torch.Generator(device=DEV)
    g.manual_seed(73)
    ids = torch.randint(-1, L, (M,), generator=g, device=DEV, dtype=torch.int32)
    x = torch.empty((M, K), dtype=torch.float16, device=DEV).normal_(generator=g)
    y = torch.empty((M, N), dtype=torch.float16, device=DEV).normal_(generator=g)
    order, offsets = fq.group_rows(ids, L)
    out = fq.adapters(to_dev(a), to_dev(b), to_dev(scale), x, order, offsets, y)
    for at in (slice(0, 40), slice(M // 2 - 20, M // 2 + 20), slice(M - 40, M)):
        want, bound = ref.adapters(a, b, scale, host(x[at]), host(ids[at]), host(y[at]))
        assert np.all(np.abs(host(out[at]).astype(np.float64) - want) <= bound)
    assert torch.equal(out[ids < 0], y[ids < 0])
