"""The block-scaled FP8 product at shapes for which each tile height (64 to 256 rows) and the strips run, whole and with the reduction
split, plain, onto a residual and with SiLU.  Reference and tolerances: tests/test_gpu_fp8_block.py, here formed in float64 on
the device (a float64 sum of K products is off by K 2^-53 of the absolute terms, which the tolerance's own K 2^-23 of them hides)."""
import pytest
import torch

from paper_2505_07203_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def outliers(g, r, k, scale):
    x = torch.randn(r, k, device="cuda", generator=g) * scale
    x[:, torch.randint(0, k, (max(1, k // 200),), device="cuda", generator=g)] *= 30.0
    return x.to(torch.bfloat16)


def values(codes, scales, block):
    s = scales.t() if block == 1 else scales.repeat_interleave(128, 0)[:codes.shape[0]]
    return codes.view(torch.float8_e4m3fn).double() * s.double().repeat_interleave(128, 1)


def sum_err(av, wv):
    top = lambda x: x.abs().reshape(x.shape[0], -1, 8).amax(2)
    return 7 * 2.0 ** -13 * (top(av) @ top(wv).t()) + av.shape[1] * 2.0 ** -23 * (av.abs() @ wv.abs().t())


# strips | 64, 128, 192, 256 rows, whole | the same with the reduction split
SHAPES = [(1, 1088, 4096), (16, 576, 2048), (17, 576, 256), (193, 8256, 256), (385, 8256, 256), (385, 14336, 256), (17, 576, 2048), (65, 6208, 4096),
          (129, 4160, 8192), (193, 6208, 8192)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_a_tile(M, N, K):
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    a, w, r = outliers(g, M, K, 1.0), outliers(g, N, K, 0.02), outliers(g, M, N, 1.0)
    qa, sa = B.po_op_quantize_blocks(a)
    qw, sw = B.po_op_quantize_blocks(w, 128)
    av, wv = values(qa, sa, 1), values(qw, sw, 128)
    ref, err = av @ wv.t(), sum_err(av, wv)
    empty = torch.empty(0, dtype=torch.uint8, device="cuda")
    for kw in ({}, {"scratch": empty}):
        for res in (None, r):
            want = ref if res is None else ref + res.double()
            got = B.po_op_linear_fp8_block(qa, sa, qw, sw, residual=res, **kw).double()
            assert bool(((got - want).abs() <= 2.0 ** -8 * (want.abs() + err) + err + 1e-30).all())


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_a_tile_with_silu(M, N, K):
    F = N // 64 * 32
    g = torch.Generator(device="cuda").manual_seed(M + N + K + 1)
    qa, sa = B.po_op_quantize_blocks(outliers(g, M, K, 1.0))
    (qg, sg), (qu, su) = (B.po_op_quantize_blocks(outliers(g, F, K, 0.02), 128) for _ in range(2))
    av, gv, uv = values(qa, sa, 1), values(qg, sg, 128), values(qu, su, 128)
    packed = B.po_op_pack_gate_up(qg.view(torch.bfloat16), qu.view(torch.bfloat16)).view(torch.uint8)
    gate, up = av @ gv.t(), av @ uv.t()
    ref = gate / (1 + torch.exp(-gate)) * up
    eg, eu = sum_err(av, gv), sum_err(av, uv)
    e = 1.1 * eg * (up.abs() + eu) + gate.abs() * eu
    tol = 2.0 ** -8 * (ref.abs() + e) + e + 2.0 ** -20 * ref.abs() + 1e-30
    for kw in ({}, {"scratch": torch.empty(0, dtype=torch.uint8, device="cuda")}):
        got = B.po_op_linear_fp8_block(qa, sa, packed, torch.stack((sg, su)), silu_mul=True, **kw).double()
        assert bool(((got - ref).abs() <= tol).all())
