"""The block-scaled FP8 product with more columns than strips of 16 make workgroups for one launch (2^24 of 256 threads)."""
import pytest
import torch

from paper_2505_07203_amd import binding as B

pytestmark = pytest.mark.gpu


def test_one_row_by_2_to_28_columns():
    """32 GiB of weights whose codes are all 1: a column is the sum of the activation's codes times its block's scale"""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    N, K = 1 << 28, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    a = torch.tensor([0x38, 0x40, 0xb8, 0x30] * 32, dtype=torch.uint8, device="cuda")[None]      # 1, 2, -1, 0.5: 80 together
    a_scales = torch.full((1, 1), 0.25, device="cuda")
    w = torch.full((N, K), 0x38, dtype=torch.uint8, device="cuda")
    w_scales = torch.rand(N // 128, 1, generator=g, device="cuda")
    w_scales = w_scales.to(torch.bfloat16).float()                                                # (products by 20 are then exact in float32)
    c = B.po_op_linear_fp8_block(a, a_scales, w, w_scales)
    want = (w_scales * 20.0).to(torch.bfloat16).expand(N // 128, 128).reshape(1, N)
    assert torch.equal(c, want)
