"""What the operators around the shared products refuse (host logic: no call here reaches a launch)."""
import ctypes as C

import numpy as np
import pytest

from paper_2505_07203_amd import binding as B

P = 0x1000            # stands for a device pointer: refused calls never look at it


def refused(f, ok, changes):
    for change in changes:
        *pairs, status = change
        a = list(ok)
        for i, v in zip(pairs[::2], pairs[1::2]):
            a[i] = v
        assert f(*a) == status, change


def test_add_rmsnorm_quantize_refusals():
    # x, delta, g, h, y, codes, scales, rows, d, block, eps, stream
    ok = [P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 7 * P, 4, 256, 128, 1e-5, None]
    refused(B.lib().po_op_add_rmsnorm_quantize, ok, [
        (0, None, 1), (2, None, 1), (4, None, 5, None, 6, None, 1), (5, None, 1), (6, None, 1), (7, 0, 1), (7, -1, 1), (8, 0, 1), (9, 1, 1), (9, 64, 1), (9, -128, 1),
        (4, 4 * P, 1), (5, P, 1), (5, 2 * P, 1), (5, 4 * P, 1), (5, 5 * P, 1), (10, -1.0, 1), (10, float("nan"), 1),
        (8, 192, 2), (8, 260, 9, 0, 2), (8, 16384 + 128, 2), (7, 1 << 24, 4)] + [(i, ok[i] + 8, 1) for i in range(6)])


def ints(*v):
    return (C.c_int32 * len(v))(*v)


def segs(*v):
    return (C.c_int64 * (3 * len(v)))(*[x for s in v for x in s])


def test_adapters_refusals():
    # dtype, x, a, b, ranks, scales, slots, width, residual, c, rows, N, K, segments, n, scratch, bytes, stream
    rk, sc, sg = ints(8, 16, 0), (C.c_float * 3)(1, 1, 1), segs((0, 4, 0), (4, 3, -1), (9, 1, 2))
    ok = [1, P, 2 * P, 3 * P, rk, sc, 3, 16, 4 * P, 5 * P, 10, 64, 128, sg, 3, 6 * P, 1 << 30, None]
    refused(B.lib().po_op_adapters, ok, [
        (0, 2, 1), (0, -1, 1), (1, None, 1), (2, None, 1), (3, None, 1), (4, None, 1), (5, None, 1), (6, 0, 1), (7, 0, 1), (7, 12, 2), (7, 136, 2), (7, 8, 1), (9, None, 1), (9, P, 1), (8, P, 1),
        (10, 0, 1), (10, 9, 1), (11, 0, 1), (11, 60, 2), (12, -8, 1), (12, 100, 2), (13, None, 1), (14, -1, 1), (15, None, 1), (15, 6 * P + 64, 1), (16, 0, 6), (6, 2, 1),
        (10, (1 << 23) + 1, 4), (11, (1 << 20) + 8, 4), (12, (1 << 17) + 8, 4), (4, ints(8, 17, 0), 1), (4, ints(-1, 16, 0), 1),
        (13, segs((0, 4, 0), (3, 3, -1), (9, 1, 2)), 1), (13, segs((0, 4, 0), (4, -1, -1), (9, 1, 2)), 1), (13, segs((0, 4, 3), (4, 3, -1), (9, 1, 2)), 1),
        (13, segs((0, 4, -2), (4, 3, -1), (9, 1, 2)), 1), (13, segs((-1, 4, 0), (4, 3, -1), (9, 1, 2)), 1), (13, segs((0, 4, 0), (4, 3, -1), (9, 2, 2)), 1),
        (13, segs((0, 4, 0), (4, 3, -1), (1 << 62, 1 << 62, 2)), 1)] + [(i, ok[i] + 8, 1) for i in (1, 2, 3, 8, 9)])
    n = C.c_size_t(7)
    f = B.lib().po_adapters_bytes
    assert f(1, rk, 3, 16, 10, 64, 128, sg, 3, None) == 1 and f(1, rk, 3, 12, 10, 64, 128, sg, 3, C.byref(n)) == 2 and n.value == 7
    assert B.po_adapters_bytes(B.PO_BF16, [8, 16, 0], 16, 10, 64, 128, [(0, 4, 0)]) < 1 << 20
    with pytest.raises(ValueError):
        B.po_adapters_bytes(B.PO_BF16, [8], 16, 10, 64, 128, np.zeros((2, 4)))


def test_token_logprobs_refusals():
    # dtype, logits, ld, rows, V, tokens, n_tokens, top, logprobs, entropy, top_tokens, top_logprobs, scratch, bytes, stream
    ok = [0, P, 1000, 4, 1000, P, 2, 5, P, P, P, P, P, 1 << 30, None]
    refused(B.lib().po_op_token_logprobs, ok, [
        (0, 2, 1), (1, None, 1), (1, P + 2, 1), (2, 999, 1), (2, -1000, 1), (3, 0, 1), (3, (1 << 20) + 1, 4), (4, 0, 1), (5, None, 1), (6, -1, 1), (7, -1, 1), (7, 65, 1), (8, None, 1),
        (10, None, 1), (11, None, 1), (12, None, 1), (12, P + 64, 1), (13, 0, 6), (13, B.po_token_logprobs_bytes(4, 1000, 5) - 1, 6), (2, 1 << 25, 4, (1 << 24) + 1, 4),
        (6, 0, 7, 0, 9, None, 1), (0, 1, 1, P + 1, 1)])
    n = C.c_size_t(7)
    f = B.lib().po_token_logprobs_bytes
    assert f(4, 1000, 0, None) == 1 and f(0, 1000, 0, C.byref(n)) == 1 and f(4, 1000, 65, C.byref(n)) == 1 and f(4, 1 << 25, 0, C.byref(n)) == 4 and n.value == 7
    for rows in (1, 3, 1000):
        for V in (1, 1000, 128256):
            assert 0 < B.po_token_logprobs_bytes(rows, V) < B.po_token_logprobs_bytes(rows, V, 20)


def test_lm_head_logprobs_refusals():
    # dtype, x, w, tokens, logprobs, entropy, rows, V, d, scratch, bytes, stream
    ok = [1, P, P, P, P, P, 4, 1000, 128, P, 1 << 40, None]
    refused(B.lib().po_op_lm_head_logprobs, ok, [
        (0, 2, 1), (1, None, 1), (2, None, 1), (1, P + 8, 1), (2, P + 8, 1), (3, None, 1), (4, None, 1), (3, None, 4, None, 5, None, 1), (6, 0, 1), (6, (1 << 20) + 1, 4), (7, 0, 1), (7, (1 << 24) + 1, 4),
        (8, 0, 1), (8, 96, 2), (0, 0, 8, 66, 2), (8, (1 << 16) + 64, 4), (9, None, 1), (9, P + 128, 1), (10, 0, 6), (10, B.po_lm_head_logprobs_bytes(1, 4, 1000, 128) - 1, 6)])
    n = C.c_size_t(7)
    f = B.lib().po_lm_head_logprobs_bytes
    assert f(1, 4, 1000, 128, None) == 1 and f(2, 4, 1000, 128, C.byref(n)) == 1 and f(1, 4, 1000, 100, C.byref(n)) == 2 and n.value == 7


def test_token_logprobs_of_too_many_tokens():
    """a row's tokens are counted in 32 bits, 256 at a time"""
    ok = [0, P, 1000, 1, 1000, P, 2, 0, P, P, None, None, P, 1 << 30, None]
    refused(B.lib().po_op_token_logprobs, ok, [(6, (1 << 30) + 1, 4), (6, (1 << 31) - 1, 4), (6, (1 << 31) - 257, 4), (6, 1 << 30, 13, 0, 6)])
