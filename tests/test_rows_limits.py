"""A launch holds fewer than 2^32 threads: calls that would need more are refused on the host."""
import ctypes

import paper_2508_04405_amd as fq

P16 = ctypes.c_void_p(0x1000)
ESHAPE = -2


def test_combine():
    f = fq.load().flexq_expert_combine
    for M, N in ((1 << 20, 1 << 15), (1 << 30, 32), (2**31 - 1, 2**31 - 32)):
        assert f(P16, P16, P16, None, M, 2, N, P16, None) == ESHAPE, (M, N)


def test_adapters():
    f = fq.load().flexq_adapters
    for M, N, R in ((1 << 24, 1 << 20, 16), (1 << 24, 1 << 20, 256), (1 << 20, 2**31 - 32, 64)):
        assert f(P16, P16, P16, 4, R, P16, P16, P16, M, N, 128, P16, P16, P16, 1 << 60, None) == ESHAPE, (M, N, R)
