"""Routing to experts on the GPU where rounding could decide: large biases, and weights to the last places of fp32."""
import numpy as np
import pytest
import torch

import paper_2508_04405_amd as fq
import rows_reference as ref
from gpu_helpers import say, to_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("size", [64.0, 256.0, 65536.0])
@pytest.mark.parametrize("E,groups,top_groups,k", [(16, 8, 3, 4), (64, 32, 9, 6), (48, 8, 2, 3), (510, 17, 5, 16)])
def test_groups_whose_large_biases_cancel(E, groups, top_groups, k, size, score):
    """A group's best two c, +size and -size and something, are good to fp32's step at `size`; what they add up to is about
    1, and differs between groups by about that step."""
    say(f"route E={E} groups={groups}/{top_groups} biases of {size} {score}")
    rng = np.random.default_rng([E, int(size)])
    each, M = E // groups, 300
    logits = np.tile(rng.standard_normal(each), groups)[None, :]
    step = size * 2.0**-20 * (1.0 if score == "sigmoid" else E / 4.0)        # a softmax's scores are as much smaller
    logits = (logits + step * rng.standard_normal((M, E))).astype(np.float32)
    bias = np.full(E, -size, np.float32)
    bias[::each] = size
    kw = dict(score=score, groups=groups, top_groups=top_groups, group_top=2)
    experts, _ = ref.route(logits, k, bias=bias, **kw)
    got = fq.route_experts(to_dev(logits), k, bias=to_dev(bias), **kw).experts.cpu().numpy()
    wrong = np.flatnonzero((got != experts).any(1))
    assert wrong.size == 0, (wrong.size, got[wrong[:3]], experts[wrong[:3]])


# ---- weights -----------------------------------------------------------------------------------------------------

def check_weights(logits, k, score, renormalise, scale=1.0, bias=None):
    """Roundings counted in 2^-24 of the value: an exponential 2 (an ulp) and what its argument was rounded by, put right, 1;
    by sigmoids 1 + e^l 2 and the quotient 1: 6.  Renormalised: sixteen added up two by two 4, on terms off by 6, the
    quotient 1, the scale 1: 18.  A softmax over all: its terms 2, their arguments' rounding 4 (their distance from the
    largest logit, by what they weigh in the sum: at most 4 for 512 experts), additions 7 + 2 + 4; the chosen one 3, quotient 1,
    scale 1: 24.  Subnormal weights: half a step of 2^-149 for the exponential, twice as much by the ulp, the product and the
    quotient each, twice all that where the sum is 1/2, times the scale, and a rounding of its own."""
    r = fq.route_experts(to_dev(logits), k, score=score, renormalise=renormalise, scale=scale,
                         bias=None if bias is None else to_dev(bias))
    experts, want = ref.route(logits, k, score, renormalise=renormalise, scale=scale, bias=bias)
    assert np.array_equal(r.experts.cpu().numpy(), experts)
    off = np.abs(r.weights.cpu().numpy().astype(np.float64) - want)
    bound = (18 if renormalise else 24) * 2.0**-24 * np.abs(want) + (6 * scale + 1) * 2.0**-149
    worst = (off / bound).max()
    say(f"    worst weight: {worst:.2f} of the bound")
    assert worst <= 1.0, (worst, np.argwhere(off > bound)[:3], want[off > bound][:3], off[off > bound][:3])


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_weights_of_distant_logits(score, renormalise):
    """Differences of logits that fp32 rounds: by 2^-24 of themselves, which are up to 100."""
    say(f"weights {score} renormalise={renormalise}")
    pairs = np.array([[0.1, 60.3], [40.7, 0.3], [-0.1, -60.3], [-40.7, -0.3], [99.9, 0.7], [-0.7, -85.1]], np.float32)
    check_weights(pairs, 2, score, renormalise)
    rng = np.random.default_rng(50)
    for E, k in ((8, 2), (64, 16), (60, 5), (512, 16)):
        for spread in (1.0, 5.0, 30.0):
            logits = (spread * rng.standard_normal((100, E))).astype(np.float32)
            zero = np.zeros(E, np.float32)
            check_weights(logits, k, score, renormalise, 2.5)
            check_weights(logits.astype(np.float16), k, score, renormalise)
            if score == "softmax" or spread < 30.0:           # (sigmoids of more are 1 in 64 bits, ties)
                check_weights(logits, k, score, renormalise, bias=zero)


def test_weights_of_even_softmaxes():
    """Many experts of about one score: the sum's additions."""
    rng = np.random.default_rng(51)
    for E in (64, 256, 511, 512):
        logits = (0.01 * rng.standard_normal((50, E))).astype(np.float32)
        logits[::2, 5] = 5.0
        for renormalise in (True, False):
            check_weights(logits, 8, "softmax", renormalise)
            check_weights(logits, 8, "softmax", renormalise, bias=np.zeros(E, np.float32))


@pytest.mark.parametrize("renormalise", [True, False])
def test_weights_of_sigmoids_far_below_zero(renormalise):
    """Scores that are subnormal in fp32, alone and beside one that is not."""
    rng = np.random.default_rng(52)
    logits = rng.uniform(-104.0, -80.0, (200, 16)).astype(np.float32)
    logits[50:100] = rng.uniform(-95.0, -86.0, (50, 16))
    logits[100:, 3] = rng.uniform(-80.0, 5.0, 100)
    check_weights(logits, 6, "sigmoid", renormalise)
    check_weights(logits, 6, "sigmoid", renormalise, 2.5)
    check_weights(logits.astype(np.float16), 6, "sigmoid", renormalise)
