"""The sizes of the GPU tests of the LM head's log-probabilities reach every tile that its launches take (the choice is a host function of sizes): a refit
of its constants that moved a tile out of the tests' sizes fails here."""
from paper_2505_07203_amd import binding as B

import test_gpu_head_logprobs_tiles as T

BF16 = {(r, 128) for r in (32, 64, 96, 128, 160, 192, 256)} | {(192, 256), (256, 256)}
PAST_CACHES = 256 << 20


def blocks(dtype, rows, V, d):
    """of columns that leave sums for each row: three numbers each, and the token's logit"""
    return (B.po_lm_head_logprobs_bytes(dtype, rows, V, d) // rows - 4) // 12


def bf16_tile(rows, V, d):
    """of the products with as many whole 64 columns"""
    assert rows > 16
    tile = B.po_gemm_tile(rows, (V + 63) // 64 * 64, d, 1)[:2]
    assert blocks(B.PO_BF16, rows, V, d) == (V + tile[1] - 1) // tile[1]
    return tile


def f32_tile(rows, V, d):
    """rows of a tile of 128 columns: as few tiles as there can be of as few times 16 rows as these need; or of 32 columns"""
    n = blocks(B.PO_F32, rows, V, d)
    assert n in ((V + 31) // 32, (V + 127) // 128)
    if n == (V + 31) // 32:
        return 32, 32
    tiles = (rows + 63) // 64
    return ((rows + tiles - 1) // tiles + 15) // 16 * 16, 128


def test_bf16():
    assert {bf16_tile(*s) for s in T.BF16} == BF16
    # several row tiles, in the smallest only where there are few columns: not among these
    assert {t for s in T.BF16 for t in [bf16_tile(*s)] if s[0] > t[0]} == BF16 - {(32, 128)}
    assert all(rows % bf16_tile(rows, V, d)[0] and V % 64 for rows, V, d in T.BF16)


def test_bf16_past_the_caches():
    assert all(V * d * 2 >= PAST_CACHES for _, V, d in T.BF16_ONCE)
    one = {bf16_tile(*s) for s in T.BF16_ONCE if s[0] > 16 and s[0] <= bf16_tile(*s)[0]}
    assert one == BF16 - {(256, 128)}                                 # (which launches of so many columns do not take)


def test_float32():
    every = {(32, 32)} | {(r, 128) for r in (16, 32, 48, 64)}
    assert {f32_tile(*s) for s in T.F32} == every
    assert {f32_tile(*s) for s in T.F32 if s[0] > 64} >= {(32, 32), (48, 128), (64, 128)}
    assert {f32_tile(*s) for s in T.F32_ONCE} == every
    assert all(V * d * 4 >= PAST_CACHES and rows <= f32_tile(rows, V, d)[0] for rows, V, d in T.F32_ONCE)
