"""The operators whose rows choose their own weights refuse wrong arguments with the library's own error, before they take
memory or touch the GPU."""
import pytest
import torch

import paper_2508_04405_amd as fq

HALF, I8 = torch.float16, torch.int8


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
