"""The experts' layers on the GPU, kernel by kernel: their bits, and outputs past 32 bits."""
import numpy as np
import pytest
import torch

import paper_2508_04405_amd as fq
from paper_2508_04405_amd import dev
import rows_reference as ref
from gpu_helpers import assert_y_close, say, to_dev
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


def test_a_forced_kernel_is_the_one_that_runs():
    """With group-128 scales too; values are compared elsewhere, up to the order of fp32 sums."""
    rng = np.random.default_rng(60)
    codes, sw = draw_experts(rng, 2, 288, 384, 128)
    xq, sx = (to_dev(v) for v in draw_rows(rng, 70, 384, 8))
    packed = fq.pack_experts(to_dev(codes), to_dev(sw), 128)
    order, offsets = fq.group_rows(torch.arange(70, dtype=torch.int32, device=DEV) % 2, 2)
    for form in range(1, 7):
        assert dev.expert_linear(form, packed, 288, 384, xq, sx, order, offsets, group=128, k=1)[1] == form
    assert 1 <= dev.expert_linear(0, packed, 288, 384, xq, sx, order, offsets, group=128, k=1)[1] <= 6


@pytest.mark.parametrize("group", [0, 128])
def test_streaming_rows_past_32_bits(group):
    """The streaming kernel on an output of more than 2^32 bytes, sorted and scattered."""
    rng = np.random.default_rng([61, group])
    E, N, K, slots = 2, 32768, 128, 70000
    codes, sw = draw_experts(rng, E, N, K, group)
    xq, sx = draw_rows(rng, slots, K, 8)
    order, offsets = ref.group_rows((np.arange(slots) % 2).astype(np.int32), E)
    args = (fq.pack_experts(to_dev(codes), to_dev(sw), group), N, K, to_dev(xq), to_dev(sx), to_dev(order), to_dev(offsets))
    at = np.array([0, 34999, 35000, 65535, 65536, 69998, 69999])            # sorted rows
    want, slack = ref.expert_rows(codes, sw, xq[order[at]], sx[order[at]], np.arange(at.size), np.array([0, 2, at.size]), 1, group)
    out = torch.empty((slots, N), dtype=torch.float16, device=DEV)
    for scatter in (False, True):
        say(f"group={group} scatter={scatter}")
        out.fill_(7.0)
        _, ran = dev.expert_linear(1, *args, group=group, k=1, scatter=scatter, out=out)
        assert ran == 1
        rows = torch.from_numpy(order[at] if scatter else at).long().to(DEV)
        assert_y_close(host(out[rows]), want.astype(np.float16), slack if group else None)
