"""The operators for batches where offsets pass 31 and 32 bits: the same numbers as on a small copy of what is used."""
import numpy as np
import pytest
import torch

from paper_2505_07203_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.empty_cache()


def rnd(seed, *shape):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(torch.bfloat16)


@pytest.mark.parametrize("hq,requests", [(4, [(0, 3, 0, 150), (3, 1, 152, 70)]), (16, [(0, 300, 0, 300), (300, 170, 304, 170)]), (8, [(0, 1, 0, 600)])])
def test_attention_rows_of_one_kv_head_more_than_2_gib_apart(hq, requests):
    """V^T of one KV head: 128 rows of 9.4 million columns; own keys at its end, the prefix in the same tensors"""
    hd, n2, cols = 128, 700, (1 << 23) + (1 << 20)
    n = max(r[2] + r[3] for r in requests)
    q, k, v = rnd(1, max(r[0] + r[1] for r in requests), hq, hd) * 0.1, rnd(2, n, 1, hd), rnd(3, hd, n)
    k2, v2 = rnd(4, n2, 1, hd), rnd(5, hd, 704)
    if n % 8:
        v = torch.cat((v, v.new_zeros(hd, 8 - n % 8)), 1)
    at = cols - 1024
    kf, vf = torch.empty(cols, 1, hd, dtype=torch.bfloat16, device="cuda"), torch.empty(hd, cols, dtype=torch.bfloat16, device="cuda")
    kf[at:at + n], vf[:, at:at + n] = k, v[:, :n]
    kf[:n2], vf[:, :n2] = k2, v2[:, :n2]
    far = [(a, b, c + at, d) for a, b, c, d in requests]
    want = B.po_op_attention_shared(q, k, v, requests, k2, v2, n2, q_prescaled=True)
    got = B.po_op_attention_shared(q, kf, vf, far, kf, vf, n2, q_prescaled=True)
    assert torch.equal(got, want)


def test_quantisation_and_product_of_more_than_2_gib_of_codes():
    M, K, N = 300_001, 8192, 64
    x = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    for i in range(0, M, 50_000):
        x[i:i + 50_000] = rnd(i, min(50_000, M - i), K)
    w = B.po_op_quantize_blocks(rnd(7, N, K), 128)
    qa, sa = B.po_op_quantize_blocks(x)
    got = B.po_op_linear_fp8_block(qa, sa, *w)
    for i in (0, 131_072, 262_100, M - 130):
        q, s = B.po_op_quantize_blocks(x[i:i + 130].clone())
        assert torch.equal(qa[i:i + 130], q) and torch.equal(sa[:, i:i + 130], s)
        whole = B.po_op_linear_fp8_block(q, s, *w, scratch=torch.empty(0, dtype=torch.uint8, device="cuda"))
        assert torch.equal(got[i:i + 130], whole)
    qb, sb = B.po_op_quantize_blocks(x, 128)
    i = M // 128 * 128
    q, s = B.po_op_quantize_blocks(x[i:].clone(), 128)
    assert torch.equal(qb[i:], q) and torch.equal(sb[-1:], s)


def test_logits_rows_far_apart():
    V, ld, rows = 32001, 1 << 30, 3
    store = torch.empty((rows - 1) * ld + V, dtype=torch.float32, device="cuda")
    z = store.as_strided((rows, V), (ld, 1))
    small = torch.randn(rows, V, device="cuda")
    for i in range(rows):
        z[i] = small[i]
    u = torch.tensor([0.3, 0.7, 0.95], device="cuda")
    f, i = lambda x: torch.full((rows,), x, device="cuda"), lambda x: torch.full((rows,), x, dtype=torch.int32, device="cuda")
    for kw in ({}, {"top_k": i(50)}, {"top_p": f(0.9)}, {"top_k": i(3000), "top_p": f(0.9)}, {"min_p": f(0.1)}, {"temperature": f(0.0)}):
        for a, b in zip(B.po_op_sample(z, u, **kw), B.po_op_sample(small, u, **kw)):
            assert torch.equal(a, b)
