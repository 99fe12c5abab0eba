"""Residual, norm and codes in one pass against the definition in float64.

h is one rounding of a float32 sum and compared bit for bit.  y: the sum of squares passes at most 64 + 10 float32 roundings a term (a
thread's 64 values, the tree above them), so 1 / sqrt of it is off by 40 * 2^-24 and y with its two products by less than E = 2^-18 of its value; its
rounding to bf16 is 2^-8.  A scale is off by E and two roundings.  A code is the rounding of a number within 2 E and three
roundings, less than 2^-16, of y * 448 / amax: it lies between the roundings of that number's ends."""
import numpy as np
import pytest
import torch

from paper_2505_07203_amd import binding as B

pytestmark = pytest.mark.gpu
E = 2.0 ** -18


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def inputs(rows, d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, d, device="cuda", generator=g) * torch.exp2(torch.randint(-20, 20, (rows, 1), device="cuda", generator=g).float())
    x[:, torch.randint(0, d, (max(1, d // 200),), device="cuda", generator=g)] *= 40
    delta = torch.randn(rows, d, device="cuda", generator=g) * x.abs().mean(1, keepdim=True)
    return x.bfloat16(), delta.bfloat16(), (1 + 0.2 * torch.randn(d, device="cuda", generator=g)).bfloat16()


def e4m3(t):
    return t.float().to(torch.float8_e4m3fn).double()


def check(x, delta, gain, block, eps, h, codes, scales, y):
    rows, d = x.shape
    want_h = x if delta is None else (x.float() + delta.float()).bfloat16()
    assert torch.equal(h, want_h)
    hd = want_h.double()
    ref = hd / torch.sqrt(hd.square().mean(1, keepdim=True) + eps) * gain.double()
    if y is not None:
        assert bool(((y.double() - ref).abs() <= (2.0 ** -8 + 2 * E) * ref.abs() + 2.0 ** -134).all())
    if codes is None:
        return
    b = ref.view(rows, -1, block or d)
    amax = b.abs().amax(-1)
    want_s = torch.where(amax > 0, amax.clamp(min=448 * 2.0 ** -126) / 448, torch.ones_like(amax))
    s = scales.t() if block else scales[:, None]
    assert bool(((s.double() - want_s).abs() <= 2 * E * want_s).all())
    t = (b / want_s[..., None]).view(rows, d)
    # (in the order of numbers; at 448 the end beyond it rounds to 448 too)
    c = codes.view(torch.float8_e4m3fn).double()
    lo, hi = e4m3((t - t.abs() * 2.0 ** -16 - 2.0 ** -30).clamp(-448, 448)), e4m3((t + t.abs() * 2.0 ** -16 + 2.0 ** -30).clamp(-448, 448))
    assert bool(((lo <= c) & (c <= hi)).all())


@pytest.mark.parametrize("rows,d,block", [(1, 8, 0), (1, 128, 128), (3, 200, 0), (2, 4096, 0), (5, 2048, 128), (17, 2056, 0), (7, 4224, 128), (130, 1024, 128), (33, 5120, 128),
                                          (3, 8192, 0), (4, 8200, 0), (3, 16384, 0), (2, 16384, 128), (1031, 640, 128), (300, 4096, 128), (4097, 256, 0)])
def test_definition(rows, d, block):
    x, delta, gain = inputs(rows, d, rows + d)
    if rows > 2:
        x[1], delta[1] = 0, 0                                       # a row of zeros
        if d >= 256:
            x[2, :128], delta[2, :128] = 0, 0                       # ... and a block
    for dl in (delta, None):
        for normed in (False, True):
            h, c, s, y = B.po_op_add_rmsnorm_quantize(x, dl, gain, 1e-5, block=block, normed=normed)
            assert (y is not None) == normed
            check(x, dl, gain, block, 1e-5, h, c, s, y)
    h, c, s, y = B.po_op_add_rmsnorm_quantize(x, delta, gain, 1e-5, block=block, normed=True, codes=False)
    assert c is None and s is None
    check(x, delta, gain, block, 1e-5, h, c, s, y)


def test_tiny_blocks():
    """amax below what both quotients need to be normal numbers"""
    x, delta, gain = inputs(4, 512, 3)
    gain[128:256] = 2.0 ** -125
    gain[256:384] = 2.0 ** -133
    h, c, s, y = B.po_op_add_rmsnorm_quantize(x, delta, gain, 1e-5, block=128, normed=True)
    check(x, delta, gain, 128, 1e-5, h, c, s, y)
    assert float(s[2].max()) == 2.0 ** -126


@pytest.mark.parametrize("block", [0, 128])
def test_in_place(block):
    x, delta, gain = inputs(37, 1536, 5)
    want = B.po_op_add_rmsnorm_quantize(x, delta, gain, 1e-6, block=block, normed=True)
    for which in (0, 1):
        a, b = x.clone(), delta.clone()
        got = B.po_op_add_rmsnorm_quantize(a, b, gain, 1e-6, block=block, normed=True, h=(a, b)[which])
        assert got[0] is (a, b)[which] and torch.equal((b, a)[which], (delta, x)[which])
        for p, q in zip(got, want):
            assert torch.equal(p, q)
    # h over x and y over delta, by the C interface; and the sum not kept
    a, b = x.clone(), delta.clone()
    c, s = torch.empty_like(want[1]), torch.empty_like(want[2])
    stream = torch.cuda.current_stream().cuda_stream
    B.check(B.lib().po_op_add_rmsnorm_quantize(a.data_ptr(), b.data_ptr(), gain.data_ptr(), a.data_ptr(), b.data_ptr(), c.data_ptr(), s.data_ptr(), 37, 1536, block, 1e-6, stream))
    for p, q in zip((a, c, s, b), want):
        assert torch.equal(p, q)
    a, y = x.clone(), torch.empty_like(x)
    B.check(B.lib().po_op_add_rmsnorm_quantize(a.data_ptr(), delta.data_ptr(), gain.data_ptr(), None, y.data_ptr(), None, None, 37, 1536, block, 1e-6, stream))
    assert torch.equal(a, x) and torch.equal(y, want[3])


def test_rows_do_not_depend_on_other_rows():
    x, delta, gain = inputs(70, 1024, 7)
    want = B.po_op_add_rmsnorm_quantize(x, delta, gain, 1e-5, block=128, normed=True)
    x[11, 5], x[12, 700], delta[40, 3] = float("nan"), float("inf"), float("-inf")
    keep = torch.tensor([i not in (11, 12, 40) for i in range(70)], device="cuda")
    got = B.po_op_add_rmsnorm_quantize(x, delta, gain, 1e-5, block=128, normed=True)
    for i, (p, q) in enumerate(zip(got, want)):
        p, q = (p[:, keep], q[:, keep]) if i == 2 else (p[keep], q[keep])
        assert torch.equal(p, q)
    one = B.po_op_add_rmsnorm_quantize(x[69:], delta[69:], gain, 1e-5, block=128, normed=True)
    assert torch.equal(one[1], want[1][69:]) and torch.equal(one[2][:, 0], want[2][:, 69])


def test_the_products_read_them():
    """what the call leaves is what the FP8 products take"""
    x, delta, gain = inputs(50, 1024, 9)
    g = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.randn(256, 1024, device="cuda", generator=g) * 0.02).bfloat16()
    h, c, s, y = B.po_op_add_rmsnorm_quantize(x, delta, gain, 1e-5, block=128, normed=True)
    wq, ws = B.po_op_quantize_blocks(w, 128)
    got = B.po_op_linear_fp8_block(c, s, wq, ws).double()
    av = c.view(torch.float8_e4m3fn).double() * s.t().double().repeat_interleave(128, 1)
    wv = wq.view(torch.float8_e4m3fn).double() * ws.double().repeat_interleave(128, 0).repeat_interleave(128, 1)
    ref, e = av @ wv.t(), 7 * 2.0 ** -13 * 128 * av.abs().amax(1, keepdim=True) * wv.abs().amax(1) + 1024 * 2.0 ** -23 * (av.abs() @ wv.abs().t())
    assert bool(((got - ref).abs() <= 2.0 ** -8 * (ref.abs() + e) + e).all())
    h, c, s, _ = B.po_op_add_rmsnorm_quantize(x, delta, gain, 1e-5)
    wq, ws = B.po_op_quantize_rows(w)
    got = B.po_op_linear_fp8(c, s, wq, ws).double()
    av, wv = c.view(torch.float8_e4m3fn).double() * s[:, None].double(), wq.view(torch.float8_e4m3fn).double() * ws[:, None].double()
    ref, e = av @ wv.t(), 7 * 2.0 ** -13 * 128 * av.abs().amax(1, keepdim=True) * wv.abs().amax(1) + 1024 * 2.0 ** -23 * (av.abs() @ wv.abs().t())
    assert bool(((got - ref).abs() <= 2.0 ** -8 * (ref.abs() + e) + e).all())


def test_refusals():
    x, delta, gain = inputs(4, 256, 1)
    for bad in (dict(x=x.float()), dict(delta=delta[:, :128].contiguous()), dict(gain=gain[:8].contiguous()), dict(x=x.t().contiguous().t()), dict(x=x.cpu())):
        a = dict(x=x, delta=delta, gain=gain) | bad
        with pytest.raises(ValueError):
            B.po_op_add_rmsnorm_quantize(a["x"], a["delta"], a["gain"], 1e-5)
    with pytest.raises(B.PoError):
        B.po_op_add_rmsnorm_quantize(x[:, :200].contiguous(), None, gain[:200].contiguous(), 1e-5, block=128)


@pytest.mark.parametrize("block", [0, 128])
def test_zeros_without_eps(block):
    """a row of zeros stays one, and says nothing about its neighbours"""
    x = torch.zeros(3, 256, device="cuda").bfloat16()
    x[1] = torch.linspace(-3, 5, 256, device="cuda").bfloat16()
    gain = torch.full((256,), 1.5, device="cuda").bfloat16()
    h, c, s, y = B.po_op_add_rmsnorm_quantize(x, None, gain, 0.0, block, normed=True)
    check(x[1:2], None, gain, block, 0.0, h[1:2], c[1:2], (s[:, 1:2] if block else s[1:2]), y[1:2])
    z = torch.tensor([0, 2], device="cuda")
    assert not c[z].any() and not y[z].any() and bool(((s[:, z] if block else s[z]) == 1).all())


@pytest.mark.parametrize("rows,d,block", [(6, 8, 0), (9, 2056, 0), (9, 1024, 128), (7, 16384, 128), (7, 8200, 0)])
def test_tiny_rows(rows, d, block):
    """rows whose squares leave the range of float32 numbers, without eps or with one as small: the definition holds as for any other"""
    g = torch.Generator(device="cuda").manual_seed(d)
    gain = (1 + 0.2 * torch.randn(d, device="cuda", generator=g)).bfloat16()
    x = torch.randn(rows, d, device="cuda", generator=g).double()
    x = (x * torch.tensor([2.0 ** -t for t in (90, 64, 75, 49, 110, 126, 2, 60, 132)], device="cuda", dtype=torch.float64)[:rows, None]).float().bfloat16()
    x[:, ::3] *= 2.0 ** -6
    for eps in (0.0, 1e-42, 1e-33, 1e-28):
        for delta in (None, x.flip(1).contiguous()):
            h, c, s, y = B.po_op_add_rmsnorm_quantize(x, delta, gain, eps, block, normed=True)
            check(x, delta, gain, block, float(np.float32(eps)), h, c, s, y)
            assert torch.equal(B.po_op_add_rmsnorm_quantize(x, delta, gain, eps, block, normed=True, codes=False)[3], y)


@pytest.mark.parametrize("rows,d,block", [(16385, 4096, 0), (16385, 4096, 128), (19001, 2048, 128), (7501, 5120, 128), (7501, 5120, 0), (4801, 8192, 0), (2403, 16384, 128), (2403, 16376, 0)])
def test_past_the_caches(rows, d, block):
    """calls that move 256 MiB or more"""
    x, delta, gain = inputs(rows, d, rows + d)
    x[-2], delta[-2] = 0, 0
    want = B.po_op_add_rmsnorm_quantize(x, delta, gain, 1e-5, block=block, normed=True)
    assert rows * d * 7 >= 256 << 20
    for r0 in range(0, rows, 4096):
        part = slice(r0, r0 + 4096)
        check(x[part], delta[part], gain, block, 1e-5, want[0][part], want[1][part], want[2][:, part] if block else want[2][part], want[3][part])
    got = B.po_op_add_rmsnorm_quantize(x, delta, gain, 1e-5, block=block)                         # the codes alone
    assert all(torch.equal(a, b) for a, b in zip(got[:3], want))
    got = B.po_op_add_rmsnorm_quantize(x, delta, gain, 1e-5, block=block, normed=True, h=x)       # in place
    assert got[0] is x and all(torch.equal(a, b) for a, b in zip(got, want))
    got = B.po_op_add_rmsnorm_quantize(x, None, gain, 1e-5, block=block, normed=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
