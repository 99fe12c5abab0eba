"""Low-rank adapters of many requests against float64 arithmetic on the same operands.

Tolerances.  T = x A^T is a float32 sum whose terms pass at most K / 32 + 64 roundings in bfloat16 (the matrix instruction's chain over steps of 32, its own
adds, sums of pieces; 2^-23 each, cuts among them) and K / 16 + 64 in float32 (four products an instruction, a quarter of K a wavefront); the
second product likewise over at most 128 terms with the scale, and with bfloat16 T is kept to 2^-16 of itself.  The result's rounding is 2^-8 of the value (bfloat16) or 2^-24."""
import numpy as np
import pytest
import torch

from paper_2505_07203_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def pool(slots, width, N, K, ranks, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    a = (torch.randn(slots, width, K, device="cuda", generator=g) / K ** 0.5).to(dtype)
    b = (torch.randn(slots, N, width, device="cuda", generator=g) * 0.3).to(dtype)
    for i, r in enumerate(ranks):                                     # the rest of a slot is not used
        a[i, r:] = float("nan")
        b[i, :, r:] = float("inf")
    return a, b


def reference(x, a, b, ranks, scales, segments, res):
    """-> value and what it may be off before its rounding"""
    rows, N = len(x), b.shape[1]
    want = torch.zeros(rows, N, dtype=torch.float64, device="cuda") if res is None else res.double()
    err = torch.zeros_like(want)
    K = x.shape[1]
    for row, n, s in segments:
        if s < 0 or n == 0 or ranks[s] == 0:
            continue
        r = ranks[s]
        xd, ad, bd = x[row:row + n].double(), a[s, :r].double(), b[s, :, :r].double()
        t, ta = xd @ ad.t(), xd.abs() @ ad.abs().t()
        et = (K / (32 if x.dtype == torch.bfloat16 else 16) + 64) * 2.0 ** -23 * ta + (2.0 ** -16 * t.abs() if x.dtype == torch.bfloat16 else 0)
        sc = float(np.float32(scales[s]))
        want[row:row + n] += sc * (t @ bd.t())
        err[row:row + n] += abs(sc) * (et @ bd.abs().t() + (r + 16) * 2.0 ** -23 * ((t.abs() + et) @ bd.abs().t()))
    return want, err + 2.0 ** -23 * want.abs()


def check(x, a, b, ranks, scales, segments, res, got):
    want, err = reference(x, a, b, ranks, scales, segments, res)
    step = 2.0 ** -8 if x.dtype == torch.bfloat16 else 2.0 ** -24
    off = (got.double() - want).abs() - (step * (want.abs() + err) + err)
    assert bool((off <= 0).all()), (float(off.max()), (off > 0).nonzero()[:4])
    if res is not None:
        used = torch.zeros(len(x), dtype=torch.bool)
        for row, n, s in segments:
            used[row:row + n] = s >= 0 and ranks[s] > 0
        assert torch.equal(got[~used.cuda()], res[~used.cuda()])


def case(rows, N, K, ranks, width, segments, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 1000)
    x = torch.randn(rows, K, device="cuda", generator=g).to(dtype)
    res = torch.randn(rows, N, device="cuda", generator=g).to(dtype)
    a, b = pool(len(ranks), width, N, K, ranks, dtype, seed)
    scales = [0.5 + 0.25 * i for i in range(len(ranks))]
    return x, a, b, ranks, scales, segments, res


SHAPES = [
    (1, 8, 8, [1], 8, [(0, 1, 0)]),
    (1, 64, 64, [8], 8, [(0, 1, 0)]),
    (1, 4096, 4096, [16], 16, [(0, 1, 0)]),
    (5, 72, 136, [3, 8], 8, [(0, 2, 1), (2, 3, 0)]),
    (16, 64, 128, [16, 16], 16, [(0, 15, 0), (15, 1, 1)]),
    (17, 136, 256, [24, 5, 0], 24, [(0, 5, 2), (5, 1, 0), (6, 0, 1), (6, 11, 1)]),
    (40, 1000, 520, [32, 64, 17], 64, [(1, 7, 0), (8, 20, 1), (30, 3, -1), (33, 6, 2)]),          # rows of nobody between and at the ends
    (130, 256, 1032, [128, 100], 128, [(0, 64, 0), (64, 66, 1)]),
    (64, 512, 1024, [16] * 64, 16, [(i, 1, 63 - i) for i in range(64)]),
    (300, 264, 264, [16, 8], 16, [(i, 1, i % 2) for i in range(300)]),                            # more requests than a launch's table
    (300, 264, 264, [16, 8], 16, [(i, 1, 0) for i in range(300)]),                                # ... of one adapter
    (257, 4096, 4096, [64], 64, [(0, 257, 0)]),
    (700, 320, 14336, [16, 32], 32, [(0, 333, 1), (333, 367, 0)]),
    (2100, 640, 512, [64, 128, 8], 128, [(0, 1000, 2), (1000, 1, 0), (1001, 1099, 1)]),
    (33, 64, 64, [16], 16, []),
    # runs of many groups of 16 rows a workgroup, their last one ragged, K not whole slices
    (20011, 64, 520, [16, 64], 64, [(0, 9000, 0), (9001, 11003, 1)]),
    (17003, 136, 1160, [128, 30], 128, [(0, 30, 1), (30, 16973, 0)]),
    (9990, 64, 4104, [8], 8, [(3, 9987, 0)]),
    (16400, 72, 2560, [32], 32, [(0, 16400, 0)]),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}w{s[4]}")
def test_definition(shape, dtype):
    c = case(*shape, dtype, seed=shape[0] + shape[1])
    x, a, b, ranks, scales, segments, res = c
    seg = np.array(segments, dtype=np.int64).reshape(-1, 3)
    got = B.po_op_adapters(x, a, b, ranks, scales, seg, residual=res)
    check(*c, got)
    none = B.po_op_adapters(x, a, b, ranks, scales, seg)
    check(x, a, b, ranks, scales, segments, None, none)
    place = res.clone()
    assert B.po_op_adapters(x, a, b, ranks, scales, seg, residual=place, out=place) is place
    assert torch.equal(place, got)
    assert torch.equal(B.po_op_adapters(x, a, b, ranks, scales, seg, residual=res), got)          # the same bits every time


def test_far_offsets():
    """a pool and rows whose offsets pass 2^31 elements"""
    slots, width, K, N = 1100, 128, 16384, 64
    a = torch.empty(slots, width, K, dtype=torch.bfloat16, device="cuda")
    b = torch.empty(slots, N, width, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    for s in (0, slots - 1):
        a[s] = (torch.randn(width, K, device="cuda", generator=g) / 128).bfloat16()
        b[s] = (torch.randn(N, width, device="cuda", generator=g) * 0.3).bfloat16()
    rows = (1 << 31) // K + 40
    x = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda")
    x[-40:] = torch.randn(40, K, device="cuda", generator=g).bfloat16()
    ranks, scales = [0] * slots, [0.0] * slots
    ranks[0], ranks[-1], scales[0], scales[-1] = 128, 120, 1.0, 0.5
    seg = [(rows - 40, 3, 0), (rows - 37, 37, slots - 1)]
    got = B.po_op_adapters(x, a, b, ranks, scales, np.array(seg))
    assert not bool(got[:-40].any())
    check(x[-40:], a, b, ranks, scales, [(0, 3, 0), (3, 37, slots - 1)], None, got[-40:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_do_not_depend_on_other_rows(dtype):
    shape = (90, 200, 520, [32, 16], 32, [(0, 50, 0), (50, 40, 1)])
    x, a, b, ranks, scales, segments, res = case(*shape, dtype)
    seg = np.array(segments)
    want = B.po_op_adapters(x, a, b, ranks, scales, seg, residual=res)
    x2, res2 = x.clone(), res.clone()
    x2[7, 3], x2[50, 100], res2[20, 9] = float("nan"), float("inf"), float("nan")
    got = B.po_op_adapters(x2, a, b, ranks, scales, seg, residual=res2)
    keep = torch.tensor([i not in (7, 20, 50) for i in range(90)], device="cuda")
    assert torch.equal(got[keep], want[keep])


def test_scratch_and_outputs():
    """what scratch held changes nothing; nothing is written past it, nor behind the output"""
    x, a, b, ranks, scales, segments, res = case(45, 264, 264, [16, 40], 40, [(3, 20, 1), (23, 9, 0)], torch.bfloat16)
    seg = np.array(segments)
    want = B.po_op_adapters(x, a, b, ranks, scales, seg, residual=res)
    need = B.po_adapters_bytes(B.PO_BF16, ranks, 40, 45, 264, 264, seg)
    for fill in (0, 255, 127):
        scratch = torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda")
        out = torch.full((50, 264), 7.0, dtype=torch.bfloat16, device="cuda")
        B.po_op_adapters(x, a, b, ranks, scales, seg, residual=res, out=out[:45], scratch=scratch[:need])
        assert torch.equal(out[:45], want) and bool((out[45:] == 7.0).all()) and bool((scratch[need:] == fill).all())


def test_captured():
    """a captured call keeps its requests, ranks and scales; replays read new rows and a slot's new contents"""
    x, a, b, ranks, scales, segments, res = case(70, 512, 1024, [16, 64], 64, [(0, 1, 0), (1, 60, 1), (61, 9, 0)], torch.bfloat16)
    seg, rk, sc = np.array(segments), np.array(ranks, dtype=np.int32), np.array(scales, dtype=np.float32)
    scratch = torch.empty(B.po_adapters_bytes(B.PO_BF16, rk, 64, 70, 512, 1024, seg), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(res)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.po_op_adapters(x, a, b, rk, sc, seg, residual=res, out=out, scratch=scratch)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.po_op_adapters(x, a, b, rk, sc, seg, residual=res, out=out, scratch=scratch)
    seg[:], rk[:], sc[:] = 0, 0, 0
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        a[0, :16].copy_(torch.randn(16, 1024, device="cuda", generator=g) / 32)
        want = B.po_op_adapters(x, a, b, ranks, scales, np.array(segments), residual=res)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_beside_a_projection():
    """onto what the projection left, and into it as its residual"""
    x, a, b, ranks, scales, segments, res = case(100, 256, 512, [16, 32], 32, [(0, 30, 0), (30, 70, 1)], torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(5)
    w = (torch.randn(256, 512, device="cuda", generator=g) * 0.04).bfloat16()
    seg = np.array(segments)
    y = B.po_op_linear(x, w, residual=res)
    want, err = reference(x, a, b, ranks, scales, segments, None)
    proj = x.double() @ w.double().t()
    eproj = (512 / 32 + 64) * 2.0 ** -23 * (x.double().abs() @ w.double().abs().t())
    after = B.po_op_adapters(x, a, b, ranks, scales, seg, residual=y, out=y).double()
    into = B.po_op_linear(x, w, residual=B.po_op_adapters(x, a, b, ranks, scales, seg, residual=res)).double()
    ref = res.double() + proj + want
    # two roundings each: of the first sum and of the whole
    for got, first in ((after, res.double() + proj), (into, res.double() + want)):
        tol = 2.0 ** -8 * (first.abs() + ref.abs()) * (1 + 2.0 ** -7) + 1.01 * (err + eproj) + 2.0 ** -22 * ref.abs()
        assert bool(((got - ref).abs() <= tol).all())


def test_refusals():
    x, a, b, ranks, scales, segments, res = case(9, 64, 64, [8], 8, [(0, 9, 0)], torch.bfloat16)
    seg = np.array(segments)
    for bad in (dict(x=x.float()), dict(a=a.float()), dict(b=b[:, :56].contiguous(), residual=res), dict(residual=res[:8].contiguous()), dict(ranks=[8, 8]), dict(scales=[]),
                dict(segments=np.zeros((1, 4))), dict(x=x.cpu()), dict(x=x.t().contiguous().t())):
        k = dict(x=x, a=a, b=b, ranks=ranks, scales=scales, segments=seg, residual=None) | bad
        with pytest.raises((ValueError, TypeError)):
            B.po_op_adapters(**k)
    for bad in (dict(segments=[(0, 10, 0)]), dict(segments=[(0, 9, 1)]), dict(ranks=[9])):
        k = dict(x=x, a=a, b=b, ranks=ranks, scales=scales, segments=seg) | bad
        with pytest.raises(B.PoError):
            B.po_op_adapters(**k)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [9, 40])
def test_rows_without_an_adapter_keep_their_zeros(rows, dtype):
    """C[r] = R[r] to the sign of a zero, where the residual is not C"""
    x, a, b, ranks, scales, segments, res = case(rows, 264, 136, [16, 0], 16, [(0, 2, 0), (3, 2, 1), (rows - 2, 1, 0)], dtype)
    res[:, ::3], res[:, 1::3] = -0.0, 0.0
    got = B.po_op_adapters(x, a, b, ranks, scales, np.array(segments), residual=res)
    check(x, a, b, ranks, scales, segments, res, got)
    kept = torch.tensor([i not in (0, 1, rows - 2) for i in range(rows)], device="cuda")
    whole = torch.int16 if dtype is torch.bfloat16 else torch.int32
    assert torch.equal(got[kept].view(whole), res[kept].view(whole))


@pytest.mark.parametrize("rows", [1, 16, 17, 100])
@pytest.mark.parametrize("rank", [2, 32, 50, 100, 128])
def test_product_with_a_is_a_float32_number(rows, rank):
    """T[0] = 1 + 2^-10 + 2^-20, T[1] = -2^-10 and R = -1: every sum of these is a float32 number, and the result 2^-20"""
    K, N = 64, 136
    x, res = torch.zeros(rows, K, device="cuda").bfloat16(), torch.full((rows, N), -1.0, device="cuda").bfloat16()
    a, b = torch.zeros(1, 128, K, device="cuda").bfloat16(), torch.zeros(1, N, 128, device="cuda").bfloat16()
    x[:, :3] = 1
    a[0, 0, :3] = torch.tensor([1.0, 2.0 ** -10, 2.0 ** -20])
    a[0, rank - 1, 0] = -(2.0 ** -10)
    b[0, :, 0] = b[0, :, rank - 1] = 1
    got = B.po_op_adapters(x, a, b, [rank], [1.0], [(0, rows, 0)], residual=res)
    assert bool((got == 2.0 ** -20).all()), got.double().abs().max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,N,K,ranks", [(8007, 4096, 14336, [64, 40]), (33003, 64, 4104, [8, 16]), (33003, 64, 4104, [24, 32]), (33003, 72, 4104, [128, 3])])
def test_past_the_caches(rows, N, K, ranks, dtype):
    """calls that move 256 MiB or more read x past the caches"""
    rows = rows if dtype is torch.bfloat16 else rows // 2
    assert rows * (K + 2 * N) * (2 if dtype is torch.bfloat16 else 4) >= 256 << 20
    segments = [(2, rows // 2, 1), (rows // 2 + 3, rows - rows // 2 - 3, 0)]
    x, a, b, ranks, scales, segments, res = case(rows, N, K, ranks, (max(ranks) + 7) // 8 * 8, segments, dtype)
    got = B.po_op_adapters(x, a, b, ranks, scales, np.array(segments), residual=res)
    check(x, a, b, ranks, scales, segments, res, got)
    assert torch.equal(B.po_op_adapters(x, a, b, ranks, scales, np.array(segments), residual=res.clone()), got)
    one = B.po_op_adapters(x, a, b, ranks, scales, np.array(segments), residual=res, out=res)
    assert one is res and torch.equal(res, got)


@pytest.mark.parametrize("rows", [1, 40])
def test_product_with_a_near_the_largest_number(rows):
    """T = (2 - 2^-7 + 2^-8 + 2^-9) 2^127, which bf16 would round to infinity, B = 2^-126 and R = -4: -2^-8"""
    K, N = 64, 136
    x, res = torch.zeros(rows, K, device="cuda").bfloat16(), torch.full((rows, N), -4.0, device="cuda").bfloat16()
    a, b = torch.zeros(1, 8, K, device="cuda").bfloat16(), torch.zeros(1, N, 8, device="cuda").bfloat16()
    x[:, :3] = 2.0 ** 64
    a[0, 0, :3] = torch.tensor([(2 - 2.0 ** -7) * 2.0 ** 63, 2.0 ** 55, 2.0 ** 54])
    b[0, :, 0] = 2.0 ** -126
    got = B.po_op_adapters(x, a, b, [1], [1.0], [(0, rows, 0)], residual=res)
    assert bool((got == -(2.0 ** -8)).all()), got
