"""The operators whose rows choose their own weights refuse wrong arguments with the library's own error, before they take
memory or touch the GPU."""
import pytest
import torch

import paper_2508_04405_amd as fq

z = torch.zeros
HALF, I32, I8, U8 = torch.float16, torch.int32, torch.int8, torch.uint8


@pytest.mark.parametrize("call", [
    lambda: fq.pack_experts(z((32, 128), dtype=I8), z((32,), dtype=HALF)),
    lambda: fq.expert_linear(z(96, dtype=U8), 32, 128, z((4, 128), dtype=I8), z(4, dtype=HALF), z(4, dtype=I32), z(2, dtype=I32)),
    lambda: fq.expert_linear(z((), dtype=U8), 32, 128, z((4, 128), dtype=I8), z(4, dtype=HALF), z(4, dtype=I32), z(2, dtype=I32)),
    lambda: fq.expert_linear(z((1, 3328), dtype=U8), 32, 128, z((), dtype=I8), z(4, dtype=HALF), z(4, dtype=I32), z(2, dtype=I32)),
    lambda: fq.combine_experts(z((4, 32), dtype=HALF), z(4, dtype=I32), z(4)),
    lambda: fq.combine_experts(z(4, dtype=HALF), z((2, 2), dtype=I32), z((2, 2))),
    lambda: fq.adapters(z((16, 128), dtype=HALF), z((32, 16), dtype=HALF), z(1), z((2, 128), dtype=HALF), z(2, dtype=I32),
                        z(2, dtype=I32), z((2, 32), dtype=HALF)),
    lambda: fq.adapters(z((1, 16, 128), dtype=HALF), z((1, 32, 16), dtype=HALF), z(1), z((2, 128), dtype=HALF), z(2, dtype=I32),
                        z(2, dtype=I32), z(64, dtype=HALF)),
    lambda: fq.route_experts(z(8), 2), lambda: fq.route_experts(z((1, 1, 8)), 2)])
def test_wrong_numbers_of_dimensions(call):
    with pytest.raises(fq.FlexQError):
        call()


@pytest.mark.gpu
@pytest.mark.parametrize("group", [True, False])
def test_experts_a_token(group):
    for M in (4, 100):
        logits = torch.zeros((M, 64), device="cuda")
        for k in (-1, 0, 17, 65, 1 << 30):
            with pytest.raises(fq.FlexQError):
                fq.route_experts(logits, k, group=group)


@pytest.mark.gpu
@pytest.mark.parametrize("group", [0, 128])
def test_packing_checks_both_operands(group):
    """The packer reads as many scales as the codes' shape has rows (and groups), of fp16."""
    E, N, K = 3, 64, 256
    codes = torch.ones((E, N, K), dtype=I8, device="cuda")
    shape = (E, N) if group == 0 else (E, N, K // 128)
    fine = torch.ones(shape, dtype=HALF, device="cuda")
    assert fq.pack_experts(codes, fine, group).shape == (E, fq.packed_bytes(N, K, group))
    other = torch.ones((E, N, K // 128) if group == 0 else (E, N), dtype=HALF, device="cuda")
    for wq, sw in ((codes, fine[:2]), (codes, fine[:, :32].contiguous()), (codes, other), (codes, fine.float()), (codes, fine.cpu()),
                   (codes.float(), fine), (codes.transpose(1, 2), fine), (codes[:0], fine[:0]), (codes[:, :40].contiguous(), fine)):
        with pytest.raises(fq.FlexQError):
            fq.pack_experts(wq, sw, group)
    with pytest.raises(fq.FlexQError):
        fq.pack_experts(codes, fine, 64)
    apart = torch.ones((E, 2 * N, K), dtype=I8, device="cuda")[:, :N]        # experts that do not follow each other
    assert torch.equal(fq.pack_experts(apart, fine, group), fq.pack_experts(codes, fine, group))
