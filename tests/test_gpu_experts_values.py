"""The experts' layers on the GPU, kernel by kernel: their bits."""
import numpy as np
import pytest
import torch

import paper_2508_04405_amd as fq
from paper_2508_04405_amd import dev
from gpu_helpers import say, to_dev
from test_gpu_rows import DEV, draw_experts, draw_rows, host

pytestmark = pytest.mark.gpu


def roundings(codes, sw, xq, sx):
    """fp16 outputs, bit for bit: the exact sum as fp32, times the fp32 product of the scales, rounded at once or to fp32
    before.  (Kernels for few rows do the one, tiles the other; the dense layer's too.)"""
    acc = (xq.astype(np.int64) @ codes.astype(np.int64).T).astype(np.float32)
    by = sx.astype(np.float32)[:, None] * sw.astype(np.float32)[None, :]
    return (acc.astype(np.float64) * by.astype(np.float64)).astype(np.float16), (acc * by).astype(np.float16)


@pytest.mark.parametrize("bits", [6, 8])
@pytest.mark.parametrize("M,N,K", [(1, 64, 128), (5, 256, 1024), (33, 4128, 256), (200, 544, 640), (300, 288, 9088)])
def test_every_kernel_to_the_last_bit(M, N, K, bits):
    """Per-channel scales, all rows with one expert: each kernel's bits, and the dense layer's on that expert's weights."""
    say(f"experts M={M} N={N} K={K} bits={bits}")
    rng = np.random.default_rng([M, N, K, bits])
    codes, sw = draw_experts(rng, 3, N, K, 0)
    xq, sx = draw_rows(rng, M, K, bits)
    once, twice = roundings(codes[1], sw[1], xq, sx)
    xq, sx = to_dev(xq), to_dev(sx)
    packed = fq.pack_experts(to_dev(codes), to_dev(sw))
    order, offsets = fq.group_rows(torch.ones((M,), dtype=torch.int32, device=DEV), 3)

    def check(y, who):
        y = host(y)
        off = (y != once) & (y != twice)
        assert not off.any(), (who, int(off.sum()), y[off][:5], once[off][:5])

    for form in range(1, 7):
        y, ran = dev.expert_linear(form, packed, N, K, xq, sx, order, offsets, k=1)
        assert ran == form
        check(y, form)
    check(fq.expert_linear(packed, N, K, xq, sx, order, offsets, k=1), "chosen")
    check((fq.gemm_w6a6 if bits == 6 else fq.gemm_w6a8)(packed[1], N, K, xq=xq, sx=sx), "dense")
