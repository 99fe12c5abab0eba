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
