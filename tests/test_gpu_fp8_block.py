"""FP8 linear layers with a scale per block of 128, against their definition in float64.

Codes and scales are single-rounding results and compared bit for bit with numpy's float32 arithmetic.  The product's
reference is the exact sum of the same codes.  Its tolerance: the matrix instruction adds the products of eight consecutive k at
a time, each cut (towards zero) to multiples of 2^-13 of the power of two under the largest of the eight -- seen on the
card: 256 * 256 - 256 * 256 + x gives x = 8 and drops x = 7.5 when the three stand in one aligned eight, and is exact down to
2^-22 when x stands in another -- so seven terms of eight may each lose 2^-13 of the largest, which (largest |a|) * (largest |w|)
bounds.  The sums of eights, blocks and scaled blocks are float32: K roundings at most of 2^-24 of a partial sum that the sum of
the absolute terms bounds, doubled for the scale products.  The result's rounding to bf16 is 2^-8 of the value.
"""
import numpy as np
import pytest
import torch

from paper_2505_07203_amd import binding as B
from paper_2505_07203_amd import inputs as I
from oracle import fp8_oracle as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def bf16_dev(x32):
    bits = I.f32_to_bf16_bits(np.ascontiguousarray(x32, dtype=np.float32))
    return torch.from_numpy(bits.view(np.int16).copy()).view(torch.bfloat16).cuda(), I.stored_to_f64(bits)


def host64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def blocks64(x, rows):
    """values [R, K] -> codes [R, K] and scales [ceil(R / rows), K / 128] by the definition, in float32 steps"""
    R, K = x.shape
    nb = -(-R // rows)
    p = np.zeros((nb * rows, K), dtype=np.float32)
    p[:R] = x
    p = p.reshape(nb, rows, K // 128, 128)
    amax = np.abs(p).max((1, 3))
    safe = np.where(amax > 0, np.maximum(amax, np.float32(448.0 * 2.0 ** -126)), np.float32(448.0)).astype(np.float32)
    inv = (np.float32(448.0) / safe).astype(np.float32)
    codes = F.e4m3_encode((p * inv[:, None, :, None]).astype(np.float32)) if hasattr(F, "e4m3_encode") else None
    if codes is None:
        codes = torch.from_numpy(p * inv[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    return codes.reshape(nb * rows, K)[:R], (safe / np.float32(448.0)).astype(np.float32)


def outliers(rng, r, k, scale=1.0):
    x = rng.standard_normal((r, k), dtype=np.float32) * np.float32(scale)
    x[:, rng.integers(0, k, max(1, k // 200))] *= 30.0
    return x


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("R,K", [(1, 128), (3, 256), (127, 384), (128, 128), (129, 640), (300, 4096), (17, 14336)])
def test_quantize_blocks_is_bit_exact(R, K, rows):
    rng = np.random.default_rng(R * 31 + K + rows)
    x = outliers(rng, R, K) * np.exp2(rng.integers(-20, 20, (R, 1))).astype(np.float32)
    x[0, :128] = 0.0                                        # (rows 1) a block of zeros
    x[-1, -128:] = 2.0 ** -130                              # ... and one whose scale would not be a normal number
    if K >= 384:
        x[:, 128:256] = 0.0
    xd, x64 = bf16_dev(x)
    ref_q, ref_s = blocks64(x64, rows)
    q, s = B.po_op_quantize_blocks(xd, rows)
    assert np.array_equal(s.cpu().numpy(), ref_s.T if rows == 1 else ref_s)
    assert np.array_equal(q.cpu().numpy() & 0x7F, ref_q & 0x7F)                   # (a zero's sign is free)
    nz = (ref_q & 0x7F) != 0
    assert np.array_equal(q.cpu().numpy()[nz], ref_q[nz])


def _operands(rng, M, N, K):
    ad, a64 = bf16_dev(outliers(rng, M, K))
    wd, w64 = bf16_dev(outliers(rng, N, K, 0.02))
    qa, sa = B.po_op_quantize_blocks(ad)
    qw, sw = B.po_op_quantize_blocks(wd, 128)
    av = F.e4m3_decode(qa.cpu().numpy()) * np.repeat(sa.cpu().numpy().T.astype(np.float64), 128, 1)
    wv = F.e4m3_decode(qw.cpu().numpy()) * np.repeat(np.repeat(sw.cpu().numpy().astype(np.float64), 128, 0)[:N], 128, 1)
    return (qa, sa, qw, sw), av, wv, a64, w64


def _sum_err(av, wv):
    top = lambda x: np.abs(x).reshape(x.shape[0], -1, 8).max(2)
    return 7 * 2.0 ** -13 * (top(av) @ top(wv).T) + av.shape[1] * 2.0 ** -23 * (np.abs(av) @ np.abs(wv).T)


def _tol(av, wv, ref):
    e = _sum_err(av, wv)
    return 2.0 ** -8 * (np.abs(ref) + e) + e + 1e-30


# every tile height, slices fewer and more than a ring holds, ragged rows and columns, splits and none
@pytest.mark.parametrize("M,N,K", [(1, 64, 128), (1, 4096, 4096), (5, 192, 256), (33, 320, 384), (64, 128, 640), (65, 448, 896),
                                   (150, 512, 14336), (300, 320, 256), (257, 1024, 1152), (1000, 4160, 512), (700, 2048, 2048),
                                   (2049, 1088, 1408), (4100, 2048, 256)])
def test_linear_fp8_block(M, N, K):
    rng = np.random.default_rng(M + N + K)
    ops, av, wv, a64, w64 = _operands(rng, M, N, K)
    ref = av @ wv.T
    whole = host64(B.po_op_linear_fp8_block(*ops, scratch=torch.empty(0, dtype=torch.uint8, device="cuda")))
    assert np.all(np.abs(whole - ref) <= _tol(av, wv, ref))
    got = B.po_op_linear_fp8_block(*ops)
    assert np.all(np.abs(host64(got) - ref) <= _tol(av, wv, ref))
    assert torch.equal(got, B.po_op_linear_fp8_block(*ops))                       # (partial sums are added in order)
    rd, r64 = bf16_dev(rng.standard_normal((M, N), dtype=np.float32))
    B.po_op_linear_fp8_block(*ops, residual=rd, out=rd)                           # in place
    assert np.all(np.abs(host64(rd) - (ref + r64)) <= _tol(av, wv, ref + r64))
    # against the unquantised product: half a step of the format per operand, 2^-4 each, of the terms
    exact = a64 @ w64.T
    assert np.all(np.abs(ref - exact) <= (2 * 2.0 ** -4 + 2.0 ** -8) * 1.02 * (np.abs(a64) @ np.abs(w64).T) + 0.01 * np.abs(exact).max())


@pytest.mark.parametrize("M,Fd,K", [(1, 32, 128), (3, 160, 256), (70, 416, 512), (513, 1056, 256), (150, 2048, 4096)])
def test_gate_up_silu_fp8_block(M, Fd, K):
    rng = np.random.default_rng(M + Fd + K)
    (qa, sa, qg, sg), av, gv, _, _ = _operands(rng, M, Fd, K)
    (_, _, qu, su), _, uv, _, _ = _operands(rng, 1, Fd, K)
    packed = B.po_op_pack_gate_up(qg.view(torch.bfloat16), qu.view(torch.bfloat16)).view(torch.uint8)
    gate, up = av @ gv.T, av @ uv.T
    ref = gate / (1 + np.exp(-gate)) * up
    # d silu <= 1.1 of an error of the gate product, |silu| <= |gate|; exp, reciprocal: a few 2^-23
    eg, eu = _sum_err(av, gv), _sum_err(av, uv)
    e = 1.1 * eg * (np.abs(up) + eu) + np.abs(gate) * eu
    tol = 2.0 ** -8 * (np.abs(ref) + e) + e + 2.0 ** -20 * np.abs(ref) + 1e-30
    for scratch in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        got = host64(B.po_op_linear_fp8_block(qa, sa, packed, torch.stack((sg, su)), silu_mul=True, scratch=scratch))
        assert np.all(np.abs(got - ref) <= tol)


def test_rows_do_not_depend_on_other_rows():
    rng = np.random.default_rng(5)
    ops, *_ = _operands(rng, 200, 512, 1024)
    ref = B.po_op_linear_fp8_block(*ops)
    q = ops[0].clone()
    s = ops[1].clone()
    q[100:] = 0x7F                                                                # NaN codes in the other rows
    s[:, 100:] = float("inf")
    got = B.po_op_linear_fp8_block(q, s, ops[2], ops[3])
    assert torch.equal(got[:100], ref[:100]) and bool(torch.isnan(got[100:].float()).all())


def test_captured_and_replayed_on_another_stream():
    rng = np.random.default_rng(6)
    xd, _ = bf16_dev(outliers(rng, 40, 2048))
    wd, _ = bf16_dev(outliers(rng, 512, 2048, 0.02))
    qw, sw = B.po_op_quantize_blocks(wd, 128)
    x = xd.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        B.po_op_linear_fp8_block(*B.po_op_quantize_blocks(x), qw, sw)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = B.po_op_linear_fp8_block(*B.po_op_quantize_blocks(x), qw, sw)
    for i in range(3):
        x.copy_(xd * (i + 1) if i else xd)
        want = B.po_op_linear_fp8_block(*B.po_op_quantize_blocks(x), qw, sw)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_binding_refuses_what_the_library_cannot_see():
    rng = np.random.default_rng(7)
    (qa, sa, qw, sw), *_ = _operands(rng, 4, 128, 256)
    for bad in ((qa, sa.t().contiguous(), qw, sw), (qa[:, :128], sa, qw, sw), (qa, sa, qw, sw.double()), (qa.cpu(), sa, qw, sw),
                (qa, sa, qw[:, :128].contiguous(), sw)):
        with pytest.raises(ValueError):
            B.po_op_linear_fp8_block(*bad)
    with pytest.raises(ValueError):
        B.po_op_linear_fp8_block(qa, sa, qw, sw, residual=torch.zeros(4, 128, device="cuda"))
