"""Log-probability and entropy through the LM head against float64 arithmetic on the same operands.

Tolerances.  A logit is a float32 sum: its terms pass at most K / 32 + 32 roundings of the matrix instruction's chain and its own adds (float32:
K / 4 + 8), 2^-23 each, of a sum that the terms' magnitudes bound: e.  A log-prob moves by at most the token's own e and the largest of the row, the
entropy, whose derivative by a logit is -p (log p + H), by the largest e times sum p |log p + H| and a second order.  The sums over the
vocabulary add what the logits' own operator does (see its tests)."""
import numpy as np
import pytest
import torch

from paper_2505_07203_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def inputs(rows, V, d, seed, dtype=torch.bfloat16, lean=6.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = (torch.randn(V, d, device="cuda", generator=g) * (1.5 / d ** 0.5)).to(dtype)
    t = torch.randint(0, V, (rows,), device="cuda", generator=g).to(torch.int32)
    x = torch.randn(rows, d, device="cuda", generator=g) + torch.rand(rows, 1, device="cuda", generator=g) * lean * w[t.long()].float() / 1.5
    return x.to(dtype), w, t


def check(x, w, t, lp, ent):
    rows, d = x.shape
    V = len(w)
    wt = w.double().t().contiguous()
    steps = (d / 32 + 32 if x.dtype == torch.bfloat16 else d / 4 + 8) * 2.0 ** -23
    for r0 in range(0, rows, 256):
        xs = x[r0:r0 + 256].double()
        l = torch.log_softmax(xs @ wt, 1)
        e = steps * (xs.abs() @ wt.abs())
        z = xs @ wt
        dd = z - z.amax(1, keepdim=True)
        p = l.exp()
        a, a2, h = (p * dd.abs()).sum(1), (p * dd * dd).sum(1), -(p * l).sum(1)
        ds = 2.0 ** -24 * (96 + 8 * a)
        emax = e.amax(1)
        if lp is not None:
            tk = t[r0:r0 + 256].long()
            ok = (tk >= 0) & (tk < V)
            at = tk.clamp(0, V - 1)[:, None]
            want, got = l.gather(1, at)[:, 0], lp[r0:r0 + 256].double()
            tol = e.gather(1, at)[:, 0] + emax + ds + 2.0 ** -23 * (want.abs() + z.gather(1, at)[:, 0].abs() + z.amax(1).abs())
            assert bool(((got - want).abs() <= tol)[ok].all()), float(((got - want).abs() - tol)[ok].max())
            assert bool((got[~ok] == -float("inf")).all())
        tol = 1.1 * emax * (p * (l + h[:, None]).abs()).sum(1) + 2 * emax ** 2 * (a2 + 1) + ds * (1 + a) + 2.0 ** -24 * (96 * a + 8 * a2 + h)
        assert bool(((ent[r0:r0 + 256].double() - h).abs() <= tol).all())


@pytest.mark.parametrize("rows,V,d", [(1, 1, 64), (1, 64, 64), (2, 63, 64), (3, 65, 128), (1, 1000, 256), (16, 1024, 256), (17, 1003, 192), (5, 32001, 512), (1, 128256, 4096), (33, 5000, 320), (64, 2048, 640),
                                      (100, 33000, 256), (150, 7777, 512), (257, 4097, 256), (300, 16384, 1024), (513, 2500, 384), (1000, 3000, 512), (2500, 1500, 128), (4100, 600, 64)])
def test_definition(rows, V, d):
    x, w, t = inputs(rows, V, d, rows + V + d)
    lp, ent = B.po_op_lm_head_logprobs(x, w, t)
    check(x, w, t, lp, ent)
    again = B.po_op_lm_head_logprobs(x, w, t)
    assert torch.equal(lp, again[0]) and torch.equal(ent, again[1])
    none, only = B.po_op_lm_head_logprobs(x, w)
    assert none is None and torch.equal(only, ent)


@pytest.mark.parametrize("rows,V,d", [(1, 1, 4), (3, 65, 68), (1, 1000, 256), (16, 1024, 256), (17, 40001, 36), (130, 33000, 64), (300, 515, 512), (1100, 260, 256)])
def test_float32(rows, V, d):
    x, w, t = inputs(rows, V, d, rows + V + d, torch.float32)
    check(x, w, t, *B.po_op_lm_head_logprobs(x, w, t))


def test_tokens_and_certainty():
    x, w, t = inputs(40, 999, 128, 3, lean=300.0)                     # tokens that take all of the weight
    t[:4] = torch.tensor([-1, 999, 2**31 - 1, -(2**31)], dtype=torch.int32)
    check(x, w, t, *B.po_op_lm_head_logprobs(x, w, t))


def test_rows_do_not_depend_on_other_rows():
    for rows, V, d in ((12, 3000, 256), (300, 3000, 256), (700, 1111, 128)):
        x, w, t = inputs(rows, V, d, 5)
        lp, ent = B.po_op_lm_head_logprobs(x, w, t)
        x[7, 3], x[3, 100] = float("nan"), float("inf")
        got = B.po_op_lm_head_logprobs(x, w, t)
        keep = torch.tensor([i not in (3, 7) for i in range(rows)], device="cuda")
        assert torch.equal(got[0][keep], lp[keep]) and torch.equal(got[1][keep], ent[keep])


def test_far_weights():
    """a head whose offsets pass 2^31 elements"""
    V, d = 530_000, 4096
    w = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    for v0 in range(0, V, 50_000):
        g = torch.Generator(device="cuda").manual_seed(v0)
        w[v0:v0 + 50_000] = (torch.randn(len(w[v0:v0 + 50_000]), d, device="cuda", generator=g) * 0.02).bfloat16()
    t = torch.tensor([0, V - 1, V - 5000], dtype=torch.int32, device="cuda")
    x = (torch.randn(3, d, device="cuda") + w[t.long()].float() * 200).bfloat16()
    lp, ent = B.po_op_lm_head_logprobs(x, w, t)
    z = torch.cat([x.double() @ w[v0:v0 + 50_000].double().t() for v0 in range(0, V, 50_000)], 1)
    l = torch.log_softmax(z, 1)
    e = (d / 32 + 33) * 2.0 ** -22 * float((x.double().abs() @ w[t.long()].double().abs().t()).max())
    assert bool(((lp.double() - l.gather(1, t.long()[:, None])[:, 0]).abs() <= e).all())


def test_scratch_and_outputs():
    x, w, t = inputs(45, 5003, 192, 8)
    want = B.po_op_lm_head_logprobs(x, w, t)
    need = B.po_lm_head_logprobs_bytes(B.PO_BF16, 45, 5003, 192)
    for fill in (0, 255, 127):
        scratch = torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda")
        got = B.po_op_lm_head_logprobs(x, w, t, scratch=scratch[:need])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool((scratch[need:] == fill).all())


@pytest.mark.parametrize("rows", [4, 300])
def test_captured(rows):
    x, w, t = inputs(rows, 4000, 256, 9)
    scratch = torch.empty(B.po_lm_head_logprobs_bytes(B.PO_BF16, rows, 4000, 256), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.po_op_lm_head_logprobs(x, w, t, scratch=scratch)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.po_op_lm_head_logprobs(x, w, t, scratch=scratch)
    for seed in (20, 21, 22):
        x.copy_(inputs(rows, 4000, 256, seed)[0])
        want = B.po_op_lm_head_logprobs(x, w, t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals():
    x, w, t = inputs(4, 300, 128, 1)
    for a in ((x.double(), w, t), (x, w.float(), t), (x, w, t.long()), (x, w, t[:2]), (x, w[:, :64].contiguous(), t), (x.cpu(), w, t), (x, w.t().contiguous().t(), t)):
        with pytest.raises((ValueError, TypeError)):
            B.po_op_lm_head_logprobs(*a)
    with pytest.raises(B.PoError):
        B.po_op_lm_head_logprobs(x[:, :96].contiguous(), w[:, :96].contiguous(), t)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,V", [(1, 300), (5, 5000), (300, 256)])
def test_logits_further_apart_than_float32(dtype, rows, V):
    """logits of -2^127 and 2^127, whose distance is no float32 number: the weight is that of the larger ones, the same each, which is
    exact but for the logarithm (2^-21 of it)"""
    x = torch.zeros(rows, 64, device="cuda", dtype=dtype)
    x[:, 5] = 2.0 ** 63
    w = torch.zeros(V, 64, device="cuda", dtype=dtype)
    w[:, 5] = -2.0 ** 64
    high = torch.arange(3, V, 7, device="cuda")
    w[high, 5] = 2.0 ** 64
    t = torch.full((rows,), 3, dtype=torch.int32, device="cuda")
    lp, ent = B.po_op_lm_head_logprobs(x, w, t)
    want = torch.full((rows,), len(high), dtype=torch.float64, device="cuda").log()
    assert bool(((lp.double() + want).abs() <= 2.0 ** -21 * want).all()) and bool(((ent.double() - want).abs() <= 2.0 ** -21 * want).all())
    lp, _ = B.po_op_lm_head_logprobs(x, w, t + 1)
    assert bool((lp < -3e38).all())


@pytest.mark.parametrize("rows,V,d", [(1, 40000, 260), (31, 33001, 100), (33, 32129, 64), (48, 33000, 4), (64, 32900, 292), (65, 33000, 96), (700, 6001, 132), (17, 31, 1028)])
def test_float32_tiles(rows, V, d):
    """every tile, odd columns and ends of K, rows up to and beyond a tile's"""
    x, w, t = inputs(rows, V, d, rows + V + d, torch.float32)
    got = B.po_op_lm_head_logprobs(x, w, t)
    check(x, w, t, *got)
    again = B.po_op_lm_head_logprobs(x, w, t)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    x2 = x.clone()
    x2[0], x2[-1, 1] = float("nan"), float("inf")
    keep = slice(1, rows - 1)
    other = B.po_op_lm_head_logprobs(x2, w, t)
    assert torch.equal(other[0][keep], got[0][keep]) and torch.equal(other[1][keep], got[1][keep])
