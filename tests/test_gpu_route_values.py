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
