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


@pytest.mark.parametrize("n,q_len,kv_len,n2,heads", [(2, 2151765, 1, 3191445, (32, 8, 128)), (64, 530799, 663537, 11307814, (4, 1, 128)),
                                                     (8, 187627, 1, 16361822, (64, 64, 128)), (20, 17039, 458, 16067298, (320, 64, 128)),
                                                     (64, 4349, 0, 655911, (512, 64, 128))])
def test_attention_shared(n, q_len, kv_len, n2, heads):
    """the prefix in pieces: the tiles' launch times the pieces, and the launch that joins them with hd / 4 threads a row and head"""
    Hq, Hkv, hd = heads
    form, pieces = B.po_attention_shared_form([(i * q_len, q_len, 0, kv_len) for i in range(n)], n2, Hq, Hkv, hd)
    if form.startswith("TILES"):
        assert (n * q_len * (Hq // Hkv) + 255) // 256 * Hkv * pieces * 256 < 1 << 32
    if form in ("SPLIT", "TILES_SPLIT") or (form == "TILES" and pieces > 1):
        assert n * q_len * Hq * (hd // 4) < 1 << 32
