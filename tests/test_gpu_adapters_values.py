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


@pytest.mark.parametrize("M,R", [(9, 16), (9, 32), (9, 48), (9, 64), (9, 256), (1200, 16), (1200, 48), (1200, 128)])
def test_infinite_rows(M, R):
    """A row whose A x is infinite: infinities of the sign that B and the scale give them, NaN where ranks disagree; the other
    rows as ever.  (M = 1200: 32 rows at a time.)"""
    say(f"adapters with infinite rows M={M} R={R}")
    case = rows_exact.draw(3, M, 2, 4096 if M > 9 else 256, 25000000 // (76 * R) // 32 * 32 + 32 if M > 9 else 96, R)
    ids, x, b = case["ids"], case["x"], case["b"]
    for l in range(2):
        case["a"][l, :, 7] = 3.0
        b[l] = np.where(b[l] == 0.0, 1.0, np.abs(b[l]))       # no 0 meets an infinity
        b[l, 1::3] *= -1.0
        b[l, 2::3, R // 2:] *= -1.0                           # ranks that disagree
    h = rows_exact.intermediate(case)
    case["y"] = y = np.zeros_like(case["y"])
    one, two, three = np.flatnonzero(ids >= 0)[:3]
    x[one, 7], x[two, 7], x[three, 7] = np.inf, -np.inf, np.nan
    got = run(case)
    for row, sign in ((one, 1.0), (two, -1.0)):
        sign = sign * float(np.sign(case["scale"][ids[row]]))
        assert np.all(got[row, 0::3] == sign * np.inf), row
        assert np.all(got[row, 1::3] == -sign * np.inf), row
        assert np.all(np.isnan(got[row, 2::3])), row
    assert np.all(np.isnan(got[three]))
    rest = np.setdiff1d(np.arange(M), [one, two, three])
    bound = np.zeros_like(got, dtype=np.float64)
    for l in range(2):
        # R additions in fp32, of the halves of h that are exact here, then half a step of fp16
        bound[ids == l] = 2 * R * 2.0**-23 * abs(float(case["scale"][l])) * (np.abs(h[ids == l]) @ np.abs(b[l].astype(np.float64)).T)
    want = rows_exact.term(case, h)
    assert np.all(np.abs(got[rest].astype(np.float64) - want[rest]) <= (bound + 2.0**-11 * np.abs(want) + 2.0**-25)[rest])
