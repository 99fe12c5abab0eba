"""What the entry points for batches behind one profile refuse (host logic: no call here reaches a launch)."""
import ctypes as C

import pytest

from paper_2505_07203_amd import binding as B

P = 0x1000            # stands for a device pointer: refused calls never look at it


def test_quantize_blocks_refusals():
    f = B.lib().po_op_quantize_blocks
    ok = [P, 2 * P, 3 * P, 4, 256, 1, None]
    for i, bad, status in ((0, None, 1), (1, None, 1), (2, None, 1), (1, P, 1), (3, 0, 1), (3, -1, 1), (4, 0, 1), (4, 200, 2), (4, 64, 2),
                           (5, 0, 1), (5, 64, 1), (3, (1 << 24) + 1, 4)):
        a = list(ok)
        a[i] = bad
        assert f(*a) == status, (i, bad)


def test_linear_fp8_block_refusals():
    f = B.lib().po_op_linear_fp8_block
    ok = [0, P, P, P, P, P, None, None, 0, 4, 128, 256, None]
    for i, bad, status in ((0, 3, 1), (0, -1, 1), (0, 1, 1), (1, None, 1), (2, None, 1), (3, None, 1), (4, None, 1), (5, None, 1),
                           (9, 0, 1), (9, -3, 1), (9, (1 << 24) + 1, 4), (10, 0, 1), (10, 96, 2), (11, 0, 1), (11, 192, 2), (11, 1 << 23, 4)):
        a = list(ok)
        a[i] = bad
        assert f(*a) == status, (i, bad)


def test_fp8_block_sizes_beyond_a_launch():
    assert B.lib().po_op_quantize_blocks(P, 2 * P, 3 * P, 1 << 24, 1 << 17, 1, None) == 4
    n = C.c_size_t(0)
    assert B.lib().po_linear_fp8_block_bytes(1 << 24, 1 << 17, 128, C.byref(n)) == 4


def test_fp8_block_operands_lie_on_16_bytes():
    f = B.lib().po_op_quantize_blocks
    for i in (0, 1):
        a = [P, 2 * P, 3 * P, 4, 256, 1, None]
        a[i] += 8
        assert f(*a) == 1
    f = B.lib().po_op_linear_fp8_block
    for i in (1, 3, 5, 6, 7):
        a = [1, P, P, P, P, P, P, P, 1 << 20, 4, 128, 256, None]
        a[i] += 8
        assert f(*a) == 1


def test_linear_fp8_block_bytes():
    n = C.c_size_t(7)
    f = B.lib().po_linear_fp8_block_bytes
    assert f(1, 4096, 4096, None) == 1 and f(0, 4096, 4096, C.byref(n)) == 1 and f(1, 100, 4096, C.byref(n)) == 2
    assert n.value == 7                                          # nothing is written on error
    for M, N, K in ((1, 64, 128), (150, 4096, 14336), (1, 4096, 4096), (8192, 28672, 4096)):
        b = B.po_linear_fp8_block_bytes(M, N, K)
        assert b % (4 * M * N) == 0 and b // (4 * M * N) <= 16 and b // (4 * M * N) != 1
    assert B.po_linear_fp8_block_bytes(8192, 28672, 4096) == 0   # tiles enough
    with pytest.raises(B.PoError):
        B.po_linear_fp8_block_bytes(1, 4096, 100)


def test_sample_refusals():
    f = B.lib().po_op_sample
    ok = [P, 1000, 4, 1000, P, None, None, None, None, P, None, P, 1 << 30, None]
    for i, bad, status in ((0, None, 1), (1, 999, 1), (1, -1000, 1), (2, 0, 1), (2, -1, 1), (2, (1 << 20) + 1, 4), (3, 0, 1), (4, None, 1), (9, None, 1),
                           (11, None, 1), (11, P + 64, 1), (12, 0, 6), (12, B.po_sample_bytes(4, 1000, False, False) - 1, 6)):
        a = list(ok)
        a[i] = bad
        assert f(*a) == status, (i, bad)
    a = list(ok)
    a[1] = a[3] = (1 << 24) + 1
    assert f(*a) == 4
    a = list(ok)
    a[12] = B.po_sample_bytes(4, 1000, False, False)
    a[6] = P                                                     # a setting that needs more of it
    assert f(*a) == 6


def test_sample_bytes():
    n = C.c_size_t(7)
    f = B.lib().po_sample_bytes
    assert f(4, 1000, 0, 0, None) == 1 and f(0, 1000, 0, 0, C.byref(n)) == 1 and f(4, 0, 0, 0, C.byref(n)) == 1 and f(4, 1 << 25, 0, 0, C.byref(n)) == 4
    assert n.value == 7
    for rows in (1, 3, 64, 256, 1000):
        for V in (1, 1000, 128256, 1 << 24):
            none, p, k = (B.po_sample_bytes(rows, V, *w) for w in ((False, False), (False, True), (True, True)))
            assert 0 < none < p == k                                      # (both filters use the same arrays)


def rows(*requests):
    return (C.c_int64 * (4 * len(requests)))(*[x for r in requests for x in r])


def attention_args(**kw):
    a = dict(dtype=1, q=P, q_rows=6, k=P, v=P, kv_rows=700, ldv=640, o=P, requests=rows((0, 5, 0, 5), (5, 1, 64, 30)), n_req=2, k2=P, v2=P, ldv2=128, n2=100, Hq=8,
             Hkv=2, hd=128, pre=1)
    a.update(kw)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 1), (dict(dtype=-1), 1), (dict(q=None), 1), (dict(o=None), 1), (dict(requests=None), 1), (dict(n_req=0), 1), (dict(n_req=-1), 1),
    (dict(k=None), 1), (dict(v=None), 1), (dict(k2=None), 1), (dict(v2=None), 1), (dict(n2=-1), 1), (dict(ldv2=96), 1), (dict(ldv2=132), 1),
    (dict(ldv=60), 1), (dict(ldv=637), 1), (dict(ldv=643), 1), (dict(Hq=0), 1), (dict(Hkv=0), 1), (dict(Hkv=3), 1), (dict(hd=96), 2), (dict(hd=256), 2), (dict(pre=2), 1),
    (dict(dtype=0, pre=1), 1), (dict(q=P + 8), 1), (dict(k2=P + 2), 1), (dict(v=P + 4), 1), (dict(n2=(1 << 24) + 1, ldv2=1 << 25), 4), (dict(ldv2=1 << 24), 4), (dict(ldv=1 << 24), 4),
    (dict(requests=rows((0, 5, 0, 5), (4, 1, 64, 30))), 1),            # rows of q overlap
    (dict(requests=rows((5, 1, 64, 30), (0, 5, 0, 5))), 1),            # ... descend
    (dict(requests=rows((0, -1, 0, 5), (5, 1, 64, 30))), 1), (dict(requests=rows((0, 5, 0, -5), (5, 1, 64, 30))), 1),
    (dict(requests=rows((0, 5, -8, 5), (5, 1, 64, 30))), 1), (dict(requests=rows((-3, 2, 0, 5), (5, 1, 64, 30))), 1),
    (dict(requests=rows((0, 5, 4, 5), (5, 1, 64, 30))), 1),            # V^T columns that no 16-byte load begins at
    (dict(requests=rows((0, 5, 0, 5), (5, 1, 632, 30))), 1),           # ... beyond the pitch
    (dict(requests=rows((0, (1 << 24) + 1, 0, 5), (1 << 25, 1, 64, 30))), 4), (dict(requests=rows((0, 5, 0, 5), (1 << 31, 1, 64, 30))), 4),
    (dict(Hq=1 << 17, Hkv=1), 4), (dict(q_rows=5), 1), (dict(q_rows=-1), 1), (dict(kv_rows=93), 1), (dict(kv_rows=-1), 1),
    (dict(dtype=0, pre=0, kv_rows=93), 1),
])
def test_attention_shared_refusals(change, status):
    a = attention_args(**change)
    assert B.lib().po_op_attention_shared(*a.values(), None, 0, None) == status
