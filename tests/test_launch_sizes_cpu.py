"""Sizes whose launch would have 2^32 threads or more, which HIP does not take: refused, or run in a form that has fewer (host logic: no
call here reaches a launch)."""
import pytest

from paper_2505_07203_amd import binding as B

P = 0x1000            # stands for a device pointer: refused calls never look at it
TOO_LONG = 4


@pytest.mark.parametrize("rows,K,block_rows", [(1 << 22, 8192, 1), (1 << 24, 2048, 1), ((1 << 22) - 100, 8192 + 128, 1), (1 << 18, 1 << 17, 1),
                                               (1 << 24, 1 << 14, 128), ((1 << 24) - 127, 1 << 14, 128)])
def test_quantize_blocks(rows, K, block_rows):
    blocks = (rows * K // 8 + 255) // 256 if block_rows == 1 else (rows + 127) // 128 * (K // 128)
    assert blocks * 256 >= 1 << 32
    assert B.lib().po_op_quantize_blocks(P, 2 * P, 3 * P, rows, K, block_rows, None) == TOO_LONG


@pytest.mark.parametrize("M,N", [(1, (1 << 31) - 64), (256, (1 << 31) - 128), (1 << 20, (1 << 20) - 64), (1 << 24, 1 << 16)])
def test_linear_fp8_block(M, N):
    """(128 columns and at most 256 rows a workgroup, the same number of workgroups on each of eight XCDs)"""
    assert (((M + 255) // 256) * ((N + 127) // 128) + 7) // 8 * 8 * 256 >= 1 << 32
    with pytest.raises(RuntimeError, match="status 4"):
        B.po_linear_fp8_block_bytes(M, N, 128)


@pytest.mark.parametrize("M,N", [(1, (1 << 31) - 2048), (256, (1 << 31) - 2048), (1 << 20, (1 << 19) - 256), (1 << 24, (1 << 15) - 128)])
def test_linear_fp8_block_below(M, N):
    assert ((M + 255) // 256) * ((N + 127) // 128) < (1 << 24) - 8
    assert B.po_linear_fp8_block_bytes(M, N, 128) == 0
