"""Log-probabilities, entropy and alternatives of rows of logits against float64 arithmetic on the same logits; ids are compared exactly.

Tolerances.  With d = l - m and weights e = exp(d): d is one float32 rounding, exp(d) as a power of 2 rounds d log2(e) and carries the constant's
own error, so a weight is off by (3 |d| + 4) 2^-24 of itself; a piece's sum adds 32 values in a lane and six levels above, and joining pieces
scales by one more weight.  So log S is off by ds = 2^-24 (64 + 8 A), A the mean of |d| over the distribution, a log-prob by ds and its own
rounding, T / S by 2^-24 (64 A + 8 A2) + ds A with A2 the mean of d^2, and the entropy by both."""
import math

import numpy as np
import pytest
import torch

from paper_2505_07203_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def reference(row, tokens, top):
    """one row, float64 -> log-probs, entropy, ids, their log-probs, tolerance of a log-prob, of the entropy"""
    l = np.where(np.isnan(row), -np.inf, row.astype(np.float64))
    if np.any(l == np.inf):
        l = np.where(l == np.inf, 0.0, -np.inf)
    m = l.max()
    if m == -np.inf:
        lp, ent, ds, dh = np.full_like(l, -np.inf), 0.0, 0.0, 0.0
    else:
        d = l - m
        e = np.exp(d)
        f = np.where(e > 0, d, 0.0)
        s = e.sum()
        a, a2 = (np.abs(f) * e).sum() / s, (f * f * e).sum() / s
        lp, ent = d - np.log(s), np.log(s) + a
        ds = 2.0 ** -24 * (64 + 8 * a)
        dh = ds * (1 + a) + 2.0 ** -24 * (64 * a + 8 * a2 + ent)
    order = np.argsort(-l, kind="stable")[:top]
    order = order[l[order] > -np.inf]
    ids = np.full(top, -1)
    ids[:len(order)] = order
    tlp = np.full(top, -np.inf)
    tlp[:len(order)] = lp[order]
    given = np.array([lp[t] if 0 <= t < len(l) else -np.inf for t in tokens])
    return given, ent, ids, tlp, ds, dh


def near(got, want, tol):
    got = got.astype(np.float64)
    want = np.where(want < -np.finfo(np.float32).max, -np.inf, want)          # (6.8e38 nats are more than a float32 holds)
    fin = np.isfinite(want)
    return np.array_equal(got[~fin], want[~fin]) and bool(np.all(np.abs(got[fin] - want[fin]) <= tol + 2.0 ** -24 * np.abs(want[fin])))


def check(z, tokens, top, **kw):
    lp, ent, ids, tlp = B.po_op_token_logprobs(z, tokens, top=top, **kw)
    torch.cuda.synchronize()
    zn = z.float().cpu().numpy()
    tk = np.zeros((len(z), 0), dtype=np.int32) if tokens is None else tokens.cpu().numpy()
    for i in range(len(z)):
        g, h, o, t, ds, dh = reference(zn[i], tk[i], top)
        assert np.array_equal(ids[i].cpu().numpy(), o), (i, ids[i], o)
        assert near(lp[i].cpu().numpy(), g, ds) and near(tlp[i].cpu().numpy(), t, ds), i
        assert abs(float(ent[i]) - h) <= dh, (i, float(ent[i]), h, dh)
    return lp, ent, ids, tlp


def logits(rows, V, seed, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(rows, V, device="cuda", generator=g) * 3
    z[:, torch.randint(0, V, (5,), device="cuda", generator=g)] += 8
    tk = torch.randint(0, V, (rows, 3), device="cuda", generator=g).to(torch.int32)
    return z.to(dtype), tk


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,V,top", [(1, 1, 1), (1, 1, 0), (3, 2, 5), (2, 7, 3), (5, 8, 8), (2, 511, 20), (3, 512, 64), (2, 513, 1), (4, 2047, 64), (2, 2048, 5), (3, 2049, 20), (2, 5000, 64),
                                        (7, 32001, 20), (2, 128256, 64), (3, 152064, 5), (40, 1000, 7), (300, 130, 2)])
def test_definition(rows, V, top, dtype):
    z, tk = logits(rows, V, rows + V + top, dtype)
    check(z, tk, top)
    check(z, None, top)


def test_long_rows():
    """more chunks than one list holds; offsets of the last row beyond 2^31 bytes"""
    z, tk = logits(1, 4_200_001, 1)
    check(z, tk, 64)
    big = torch.zeros(70, 8_388_608, device="cuda", dtype=torch.float32)
    big[69].copy_(logits(1, 8_388_608, 2)[0][0])
    tk = torch.tensor([[5], [8_388_607]], dtype=torch.int32, device="cuda")
    got = B.po_op_token_logprobs(big, torch.cat([tk[:1]] * 69 + [tk[1:]]), top=3)
    g, h, o, t, ds, dh = reference(big[69].cpu().numpy(), [8_388_607], 3)
    assert np.array_equal(got[2][69].cpu().numpy(), o) and near(got[0][69].cpu().numpy(), g, ds) and abs(float(got[1][69]) - h) <= dh
    assert got[2][68].tolist() == [0, 1, 2] and abs(float(got[1][68]) - math.log(8_388_608)) <= 2.0 ** -24 * 80


@pytest.mark.parametrize("top", [1, 20, 64])
def test_equal_logits(top):
    """ties by index, in rows that hold little else"""
    V = 20_000
    z = torch.zeros(6, V, device="cuda")
    z[1] = -3.5
    z[2, ::2] = 1.0
    z[3] = torch.arange(V, device="cuda").float() / 512
    z[4] = -torch.arange(V, device="cuda").float() / 512
    z[5] = (torch.arange(V, device="cuda") % 3).float() * -0.0        # -0 and 0 are equal
    check(z, torch.tensor([[0, 1, V - 1]] * 6, dtype=torch.int32, device="cuda"), top)
    check(z.bfloat16(), None, top)


def test_infinities_and_nan():
    z, tk = logits(12, 9000, 4)
    inf, nan = float("inf"), float("nan")
    z[0] = -inf
    z[1] = nan
    z[2, 5:] = -inf
    z[3, :8999] = -inf
    z[4, 100] = inf
    z[5, [7, 8000, 3000]] = inf
    z[5, 9] = nan
    z[6, ::2] = nan
    z[7, 1::2] = -inf
    z[8] = inf
    z[9, 4000:6000] = -inf
    z[10] = -3.4e38
    z[10, 77] = 3.4e38
    z[11, :] = -3.3895e38                                             # the lowest of a type as a mask
    z[11, 4], z[11, 8000] = 1.0, 2.0
    tk[2, 0], tk[2, 1], tk[4, 0], tk[5, 0], tk[5, 1], tk[6, 0], tk[6, 1] = 0, 6, 100, 8000, 1, 2, 3
    tk[7] = torch.tensor([-1, 9000, 2**31 - 1], dtype=torch.int32)
    tk[8] = torch.tensor([-(2**31), 0, 8999], dtype=torch.int32)
    for top in (0, 1, 7, 64):
        check(z, tk, top)
    check(z.bfloat16(), tk, 20)


def test_a_certain_token():
    """the rest of the distribution is far below the first token's rounding"""
    z, tk = logits(4, 3000, 6)
    for i, up in enumerate((20.0, 60.0, 150.0, 1e4)):
        z[i, 1234] = float(z[i].max()) + up
    tk[:, 0] = 1234
    check(z, tk, 4)


def test_strides():
    g = torch.Generator(device="cuda").manual_seed(8)
    for dtype in (torch.float32, torch.bfloat16):
        base = (torch.randn(5, 3333, device="cuda", generator=g) * 3).to(dtype)
        base[:, 3000:] = 100.0                                       # what lies beyond V is not used
        tk = torch.randint(0, 3000, (5, 2), device="cuda", generator=g).to(torch.int32)
        for off in (0, 1, 3, 4):
            view = base[:, off:3000 if off else 2999]
            check(view, tk.clamp(max=view.shape[1] - 1), 9)
        check(base[1:2, 5:2900], tk[:1].clamp(max=2800), 3)
        check(base[::2, :3000], tk[::2].contiguous(), 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_long_rows(dtype):
    """rows that a workgroup each reads and answers: the bits of the same rows by themselves, which are held to the definition"""
    V = 66_001
    z, tk = logits(12, V, 12, dtype)
    z[1] = -float("inf")
    z[2, 100:] = -float("inf")
    z[3] = 2.5
    z[4, [7, 60_000]] = float("inf")
    z[5, ::3] = float("nan")
    z[6] = (torch.arange(V, device="cuda") // 700).to(dtype)
    tk[7] = torch.tensor([-1, V, 0], dtype=torch.int32)
    for top in (0, 1, 20, 64):
        want = check(z, tk, top)
        for rows in (768, 1000):
            pick = torch.arange(rows, device="cuda") * 7 % 12
            got = B.po_op_token_logprobs(z[pick], tk[pick], top=top)
            assert all(torch.equal(a, b[pick]) for a, b in zip(got, want))
    odd = torch.cat((z, z[:, :3]), 1)[:, 1:V + 1]                     # a pitch that is no multiple of 16 bytes
    pick = torch.arange(800, device="cuda") % 12
    base = torch.empty(800, V + 4, dtype=dtype, device="cuda")
    base[:, 1:V + 1] = odd[pick]
    want = B.po_op_token_logprobs(odd.contiguous(), tk, top=9)
    got = B.po_op_token_logprobs(base[:, 1:V + 1], tk[pick], top=9)
    assert all(torch.equal(a, b[pick]) for a, b in zip(got, want))


def test_scratch_and_neighbours():
    """what scratch held changes nothing, nor does a neighbour; nothing is written past the outputs"""
    z, tk = logits(9, 5001, 10)
    want = B.po_op_token_logprobs(z, tk, top=20)
    for fill in (0, 255, 127):
        scratch = torch.full((B.po_token_logprobs_bytes(9, 5001, 20) + 256,), fill, dtype=torch.uint8, device="cuda")
        got = B.po_op_token_logprobs(z, tk, top=20, scratch=scratch[:-256])
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool((scratch[-256:] == fill).all())
    for i in (0, 4, 8):
        one = B.po_op_token_logprobs(z[i:i + 1], tk[i:i + 1], top=20)
        assert all(torch.equal(a[0], b[i]) for a, b in zip(one, want))
    part = B.po_op_token_logprobs(z, tk, top=5)
    assert torch.equal(part[2], want[2][:, :5].contiguous()) and torch.equal(part[1], want[1])


def test_captured():
    z, tk = logits(6, 40_000, 11)
    scratch = torch.empty(B.po_token_logprobs_bytes(6, 40_000, 20), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.po_op_token_logprobs(z, tk, top=20, scratch=scratch)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.po_op_token_logprobs(z, tk, top=20, scratch=scratch)
    for seed in (20, 21, 22):
        z.copy_(logits(6, 40_000, seed)[0])
        want = B.po_op_token_logprobs(z, tk, top=20)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    z, tk = logits(4, 300, 1)
    for a in ((z.double(), tk), (z, tk.long()), (z, tk[:2]), (z.t(), tk), (z.cpu(), tk), (z[:1].expand(4, 300), tk)):
        with pytest.raises((ValueError, TypeError)):
            B.po_op_token_logprobs(*a)
    with pytest.raises(B.PoError):
        B.po_op_token_logprobs(z, tk, top=65)
    with pytest.raises(B.PoError):
        B.po_op_token_logprobs(z, tk, top=3, scratch=torch.empty(B.po_token_logprobs_bytes(4, 300, 3) - 1, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 1500, 20_000, 131_073, 300_001])
@pytest.mark.parametrize("top", [1, 7, 32, 33, 64])
def test_where_the_answer_lies(V, top, dtype):
    """in few chunks or many, among few elements as large or thousands, at the ends of what the type holds"""
    lowest, inf = torch.finfo(dtype).min, float("inf")
    i = torch.arange(V, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(V + top)
    rows = [i / V, -i / V, (i % 2) * 3.0, (i % 511 == 17) * 2.0 - 50, torch.full((V,), lowest, device="cuda"), -1e-3 - (i // 9) * 1e-5,
            torch.where(i % 3 == 0, 0.0, -0.0), torch.where(i % 5 == 0, 1e-39, -1e-39), torch.where(i < V - 9, -inf, i / V), torch.where(i % 97 == 5, -1e30, -inf)]
    for n in (top - 1, top, top + 1):
        few = torch.full((V,), -inf, device="cuda")
        few[torch.randperm(V, device="cuda", generator=g)[:n]] = torch.randn(min(n, V), device="cuda", generator=g)
        rows.append(few)
    rows.append(torch.where(i % 1024 < 600, 5.0, torch.randn(V, device="cuda", generator=g)))
    z = torch.stack([r.float() for r in rows]).to(dtype)
    check(z, torch.randint(0, V, (len(rows), 2), dtype=torch.int32, device="cuda", generator=g), top)


@pytest.mark.parametrize("at", [0.0, 37.7, -911.3, 65_000.3, 1.04e6, -1.05e6, 3e7, -7e30])
def test_far_from_zero(at):
    """logits around a large one: distances are exact differences of float32 numbers whatever their size"""
    g = torch.Generator(device="cuda").manual_seed(7)
    z = at + torch.randn(5, 9000, device="cuda", generator=g) * max(3.0, abs(at) * 2.0 ** -22)
    check(z, torch.randint(0, 9000, (5, 3), dtype=torch.int32, device="cuda", generator=g), 9)


SIGNALLING = {torch.float32: (0x7fa00000, -0x600000, 0x7f800001), torch.bfloat16: (0x7fa0, -0x60, 0x7f81)}


def signalling(V, dtype, seed):
    """eight rows: the largest logits with a signalling NaN behind each among a lane's eight (whose larger one would be NaN), as large as others or
    300 above them; little but such NaNs; random bits"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = logits(8, V, seed, dtype)[0]
    whole = torch.int32 if dtype is torch.float32 else torch.int16
    bits = z.view(whole)
    bits[7] = torch.randint(-(2 ** 31), 2 ** 31, (V,), device="cuda", generator=g).to(whole)
    bits[6, torch.rand(V, device="cuda", generator=g) < 0.9] = SIGNALLING[dtype][2]
    for i in range(6):
        runs = torch.randperm(V // 8, device="cuda", generator=g)[:7] * 8
        for e in range(len(runs)):
            z[i, runs[e] + e] = (12.0 if i % 2 else 312.0) + e
            bits[i, runs[e] + e + 1] = SIGNALLING[dtype][(i + e) % 3]
    return z, torch.randint(0, V, (8, 3), dtype=torch.int32, device="cuda", generator=g)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [64, 700, 1200, 20_000, 40_003, 70_001, 128_256])
def test_signalling_nans(V, dtype):
    """as memory that nobody wrote may hold them: none hides a larger logit, whichever way the rows go"""
    z, tk = signalling(V, dtype, V)
    with np.errstate(invalid="ignore"):
        for top in (0, 1, 7, 40):
            want = check(z, tk, top)
            rows = 600 if V < 60_000 else 1500 if dtype is torch.float32 and V < 100_000 else 20
            pick = torch.arange(rows, device="cuda") * 3 % 8
            got = B.po_op_token_logprobs(z[pick], tk[pick], top=top)
            assert all(torch.equal(a, b[pick]) for a, b in zip(got, want))
        odd = torch.empty(8, V + 5, dtype=dtype, device="cuda")           # rows that are read one by one
        odd[:, 3:3 + V].view(torch.int32 if dtype is torch.float32 else torch.int16).copy_(z.view(torch.int32 if dtype is torch.float32 else torch.int16))
        got, want = B.po_op_token_logprobs(odd[:, 3:3 + V], tk, top=9), B.po_op_token_logprobs(z, tk, top=9)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def kinds(V, dtype):
    """twelve rows of every kind: ordinary, without weight, with few tokens, equal, infinite, with NaN, in steps"""
    z, tk = logits(12, V, 12, dtype)
    z[1] = -float("inf")
    z[2, 100:] = -float("inf")
    z[3] = 2.5
    z[4, [7, V - 300]] = float("inf")
    z[5, ::3] = float("nan")
    z[6] = (torch.arange(V, device="cuda") // 700).to(dtype)
    z[8, V - 1] = 60.0
    tk[7], tk[8] = torch.tensor([-1, V, 0], dtype=torch.int32), torch.tensor([V - 1, 0, 1], dtype=torch.int32)
    return z, tk


@pytest.mark.parametrize("V,rows", [(66_001, 1500), (524_288, 200), (524_281, 189), (130_000, 750)])
def test_long_rows_in_one_launch(V, rows):
    """float32 rows of 33 to 256 pieces, of which 48000 and more are read and answered by a workgroup a row: the bits of the same rows twelve at a time,
    which are held to the definition; aligned, and with a pitch that is no multiple of 16 bytes"""
    assert rows * ((V + 2047) // 2048) >= 48000
    z, tk = kinds(V, torch.float32)
    pick = torch.arange(rows, device="cuda") * 7 % 12
    many = z[pick]
    odd = torch.empty(rows, V + 5, device="cuda")
    odd[:, 1:V + 1] = many
    for top in (0, 1, 20, 64):
        want = check(z, tk, top)
        for rows_of in (many, odd[:, 1:V + 1]):
            got = B.po_op_token_logprobs(rows_of, tk[pick], top=top)
            assert all(torch.equal(a, b[pick]) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,rows", [(900, 513), (1003, 800), (40_000, 600), (65_536, 513), (65_536, 512), (65_537, 512), (70_001, 300)])
def test_rows_on_either_side_of_one_launch(V, rows, dtype):
    """short rows, of which more than 512 take two launches; rows above 2^16 logits"""
    z, tk = kinds(V, dtype)
    pick = torch.arange(rows, device="cuda") * 5 % 12
    many = z[pick]
    odd = torch.empty(rows, V + 5, dtype=dtype, device="cuda")
    odd[:, 1:V + 1] = many
    for top in (0, 1, 20, 64):
        want = check(z, tk, top)
        for rows_of in (many, odd[:, 1:V + 1]):
            got = B.po_op_token_logprobs(rows_of, tk[pick], top=top)
            assert all(torch.equal(a, b[pick]) for a, b in zip(got, want))
