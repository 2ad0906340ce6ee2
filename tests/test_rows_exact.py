"""That the exact adapter cases (rows_exact) tell a wrong kernel from a right one: mistakes are made in the oracle."""
import numpy as np
import pytest

import rows_exact

CASES = [(1, 1, 128, 96, 16), (5, 2, 28672, 96, 32), (40, 30, 1152, 544, 48), (100, 2, 8192, 96, 64), (100, 2, 8192, 96, 128),
         (17, 2, 640, 160, 256)]


@pytest.mark.parametrize("M,L,K,N,R", CASES)
def test_mistakes_show(M, L, K, N, R):
    case = rows_exact.draw(1, M, L, K, N, R)
    h, mine = rows_exact.intermediate(case), case["ids"] >= 0
    assert np.array_equal(rows_exact.result(case, h), case["want"])
    assert np.abs(h[mine]).max() > 2**13                      # more bits than fp16 has
    for name, wrong in (("fp16 alone", rows_exact.halved(h)), ("a step of 64 k left out", rows_exact.intermediate(case, K // 64 - 1)),
                        ("the last eighth of K left out", rows_exact.intermediate(case, K // 64 - max(1, K // 512)))):
        off = rows_exact.result(case, wrong)[mine] != case["want"][mine]
        assert off.any(1).all(), (name, "a row does not show it")
        assert off.mean() > 0.5, (name, off.mean())


def test_every_rank_counts():
    """Each rank of a lone row, left out, changes the row."""
    case = rows_exact.draw(2, 1, 1, 640, 544, 48)
    h = rows_exact.intermediate(case)
    for r in range(48):
        if h[0, r] != 0:
            one = h.copy()
            one[0, r] = 0.0
            assert (rows_exact.result(case, one) != case["want"]).any(), r
