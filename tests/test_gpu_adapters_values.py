"""Low-rank adapters on the GPU where the right answer is known to the last bit."""
import numpy as np
import pytest
import torch

import paper_2508_04405_amd as fq
import rows_exact
from gpu_helpers import say, to_dev

pytestmark = pytest.mark.gpu


def run(case, in_place=False):
    order, offsets = fq.group_rows(to_dev(case["ids"]), case["a"].shape[0])
    y = to_dev(case["y"])
    return fq.adapters(*(to_dev(case[n]) for n in ("a", "b", "scale", "x")), order, offsets, y, out=y if in_place else None).cpu().numpy()


@pytest.mark.parametrize("M,L,K,N,R", [
    (1, 1, 128, 96, 16), (1, 1, 4096, 4096, 16), (5, 2, 28672, 96, 32), (5, 2, 28672, 96, 256), (40, 30, 1152, 544, 48),
    (17, 2, 640, 160, 256), (150, 4, 384, 1056, 80), (48, 32, 8192, 1056, 64), (333, 5, 5248, 352, 32), (100, 2, 8192, 96, 16),
    (100, 2, 8192, 96, 48), (100, 2, 8192, 96, 64), (100, 2, 8192, 96, 128), (100, 2, 8192, 96, 144),
    # so many that both launches take 32 rows at a time
    (1200, 2, 4096, 20608, 16), (1200, 2, 4096, 10304, 32), (1200, 2, 4096, 6912, 48), (1200, 2, 4096, 5152, 64),
    (1200, 2, 4096, 2976, 112), (1200, 2, 4096, 2592, 128)])
def test_exact(M, L, K, N, R):
    """Bit for bit: every split and step of K, every rank, and the intermediate's bits beyond fp16's."""
    say(f"adapters M={M} L={L} K={K} N={N} R={R}")
    for seed in (1, 2):
        case = rows_exact.draw(seed, M, L, K, N, R)
        for in_place in (False, True):
            got = run(case, in_place)
            assert np.array_equal(got, case["want"]), int((got != case["want"]).sum())
