"""Attention of a batch of requests behind one shared prefix against its definition in float64.

Tolerance, per output (row, head, dimension): with a = sum p |v| / sum p over the keys the row sees,
  bf16: each probability is rounded once to bf16 for the matrix instruction, 2^-8 of it, so 2^-8 a; the result is rounded, 2^-8 of it;
  both: a score is a float32 sum of head_dim exact products, off by at most head_dim 2^-24 sum |q k|, once in the numerator and
        once in the denominator; the exponential's argument is rounded (2^-24 of up to 1.5 times the score range) and the
        exponential itself is good to 2^-22; sums over n keys round n times, 2^-24 each.
"""
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


NAN = float("nan")


class Batch:
    """inputs of a call; everything that must not be read or written holds NaN or a mark"""

    def __init__(self, seed, dtype, hq, hkv, hd, requests, n2, std=1.0, pre=True, k_rows=None):
        g = torch.Generator().manual_seed(seed)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.hq, self.hkv, self.hd, self.n2, self.pre = hq, hkv, hd, n2, pre and dtype == "bf16"
        self.req = np.array(requests, dtype=np.int64).reshape(-1, 4)
        rows = int((self.req[:, 0] + self.req[:, 1]).max()) + 3
        keys = max(int((self.req[:, 2] + self.req[:, 3]).max()) + 5, k_rows or 0)
        keys = (keys + 7) // 8 * 8
        n2c = max((n2 + 7) // 8 * 8, 8)
        rnd = lambda *s: (torch.randn(*s, generator=g) * std).to(self.dt)
        self.q = rnd(rows, hq, hd)
        if self.pre:
            self.q = (self.q.float() * B.attention_q_scale(hd)).to(self.dt)
        k, v = rnd(keys, hkv, hd), rnd(keys, hkv, hd)
        used = torch.zeros(keys, dtype=torch.bool)
        for _, nq, k0, nk in self.req.tolist():
            used[k0:k0 + nk] |= nq > 0
        k[~used] = NAN
        v[~used] = NAN
        k2, v2 = rnd(n2c, hkv, hd), rnd(n2c, hkv, hd)
        k2[n2:] = NAN
        v2[n2:] = NAN
        self.k, self.v, self.k2, self.v2 = k, v, k2, v2

    def device(self):
        lay = (lambda a: a.reshape(a.shape[0], -1).t().contiguous()) if self.dt == torch.bfloat16 else (lambda a: a)
        return [a.cuda() for a in (self.q, self.k, lay(self.v), self.k2, lay(self.v2))]

    def reference(self):
        """-> o, tolerance (float64, rows of requests only, NaN elsewhere)"""
        q, k, v, k2, v2 = (a.double() for a in (self.q, self.k, self.v, self.k2, self.v2))
        factor = math.log(2.0) if self.pre else 1.0 / math.sqrt(self.hd)
        o, tol = torch.full_like(q, NAN), torch.full_like(q, NAN)
        group = self.hq // self.hkv
        low = self.dt == torch.bfloat16
        for q0, nq, k0, nk in self.req.tolist():
            if nq == 0:
                continue
            hide = torch.arange(self.n2 + nk)[None] >= (torch.arange(nq) + self.n2 + nk - nq + 1).clamp(min=self.n2)[:, None]
            for h in range(self.hq):
                c = h // group
                kk, vv = torch.cat((k2[:self.n2, c], k[k0:k0 + nk, c])), torch.cat((v2[:self.n2, c], v[k0:k0 + nk, c]))
                qq = q[q0:q0 + nq, h]
                s = (qq @ kk.t() * factor).masked_fill(hide, -math.inf)
                top = s.amax(1, keepdim=True) if s.shape[1] else torch.zeros(nq, 1, dtype=torch.float64)
                top = torch.where(top == -math.inf, torch.zeros_like(top), top)
                p = torch.exp(s - top)
                l = p.sum(1, keepdim=True)
                l = torch.where(l == 0, torch.ones_like(l), l)
                o[q0:q0 + nq, h] = p @ vv / l
                a = p @ vv.abs() / l
                es = self.hd * 2.0 ** -24 * ((qq.abs() @ kk.abs().t()) * factor).masked_fill(hide, 0.0)
                es = es.amax(1, keepdim=True) if s.shape[1] else torch.zeros_like(l)
                span = (s.masked_fill(hide, 0.0).abs().amax(1, keepdim=True) if s.shape[1] else torch.zeros_like(l))
                rel = 2 * torch.expm1(es + 3 * span * 2.0 ** -24) + 2 * 2.0 ** -22 + 2 * (self.n2 + nk) * 2.0 ** -24
                tol[q0:q0 + nq, h] = (rel + (2.0 ** -8 if low else 0.0)) * a
        e = 2.0 ** -8 if low else 2.0 ** -24
        return o, tol * (1 + e) + e * o.abs()

    def check(self, in_place=False):
        q, k, v, k2, v2 = self.device()
        mark = q.clone() if in_place else torch.full_like(q, 777.0)
        out = q if in_place else mark.clone()
        got = B.po_op_attention_shared(q, k, v, self.req, k2, v2, self.n2, out=out, q_prescaled=self.pre)
        assert got.data_ptr() == out.data_ptr()
        want, tol = self.reference()
        asked = ~torch.isnan(want[:, 0, 0])
        d = (got.cpu().double() - want).abs()[asked]
        bad = ~(d <= tol[asked])
        assert not bad.any(), (int(bad.sum()), float((d / tol[asked]).nan_to_num(nan=math.inf).max()))
        assert torch.equal(got.cpu()[~asked], mark.cpu()[~asked])          # rows of no request
        return got


HEADS = [("bf16", 4, 2, 64), ("bf16", 8, 2, 128), ("bf16", 5, 1, 128), ("bf16", 3, 3, 64), ("f32", 4, 2, 64), ("f32", 8, 2, 128), ("f32", 5, 1, 128)]


def posts(lens, align=64, at=0):
    out, row = [], at
    for n in lens:
        out.append((row, n, row, n))
        row += (n + align - 1) // align * align
    return out


def singles(hist, align=8):
    out, row = [], 0
    for i, n in enumerate(hist):
        out.append((i, 1, row, n))
        row += (n + align - 1) // align * align
    return out


CASES = {
    "one token, no prefix": (singles([1]), 0),
    "one token behind one key": (singles([1]), 1),
    "one request": (posts([77]), 0),
    "one request behind a prefix": (posts([77]), 200),
    "posts of all lengths": (posts([1, 2, 31, 32, 33, 63, 64, 65, 100, 129]), 131),
    "posts behind whole tiles": (posts([40, 7, 90]), 256),
    "posts behind 64": (posts([40, 7]), 64),
    "tokens with histories": (singles([1, 2, 31, 32, 33, 64, 100, 257, 700]), 300),
    "tokens with histories alone": (singles([1, 8, 31, 40, 500]), 0),
    "tokens with nothing but the prefix": ([(0, 1, 0, 0), (1, 1, 0, 0), (5, 3, 0, 0)], 95),
    "empty requests among others": ([(0, 0, 0, 0), (0, 3, 0, 3), (3, 0, 8, 40), (3, 2, 8, 40), (9, 0, 48, 0)], 33),
    "rows before the first own key": ([(0, 9, 0, 4), (9, 70, 8, 66)], 0),
    "rows before the first own key, behind a prefix": ([(0, 9, 0, 4), (9, 70, 8, 66), (100, 40, 80, 0)], 17),
    "nothing to see": ([(0, 5, 0, 0), (5, 2, 0, 1)], 0),
    "several rows with a history": ([(0, 4, 0, 50), (4, 17, 56, 300), (30, 130, 360, 190)], 70),
    "shared own keys": ([(0, 3, 0, 60), (3, 1, 0, 60), (4, 40, 8, 44)], 40),
    "a long prefix": (posts([3, 20]), 5003),
    "a long prefix, tokens": (singles([3, 20, 1, 1]), 5003),
}


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("dtype,hq,hkv,hd", HEADS)
def test_against_float64(dtype, hq, hkv, hd, name):
    req, n2 = CASES[name]
    Batch(len(name) + hd, dtype, hq, hkv, hd, req, n2).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_plain_queries_and_in_place(dtype):
    Batch(3, dtype, 8, 2, 128, posts([50, 9, 140]), 333, pre=False).check(in_place=True)
    Batch(4, dtype, 4, 2, 64, singles([50, 9, 140]), 333, pre=False).check(in_place=True)
    Batch(5, dtype, 8, 2, 128, posts([50, 9, 140]), 333).check(in_place=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("std", [6.0, 0.01])
def test_scores_far_apart_and_all_alike(dtype, std):
    Batch(6, dtype, 8, 2, 128, posts([60, 3]), 700, std=std).check()
    Batch(7, dtype, 8, 2, 128, singles([60, 3]), 700, std=std).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("where", ["first", "last", "own"])
def test_one_key_far_above_the_rest(dtype, where):
    for req in (posts([50, 200]), singles([40, 7])):
        b = Batch(8, dtype, 8, 2, 128, req, 1500)
        # along every query: its score is 150 nats or more above the others
        b.q[..., 0] = 4.0
        t = 300.0 / 4.0 if b.pre else 300.0 * math.sqrt(128) / 4.0
        if where == "own":
            for _, nq, k0, nk in b.req.tolist():
                b.k[k0, :, 0] = t
        else:
            b.k2[0 if where == "first" else 1499, :, 0] = t
        b.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_requests_than_a_launch_holds(dtype):
    rng = np.random.default_rng(9)
    Batch(9, dtype, 4, 2, 64, singles(rng.integers(1, 40, 300).tolist()), 200).check()
    Batch(10, dtype, 4, 2, 64, posts(rng.integers(0, 40, 200).tolist()), 100).check()


def test_rows_do_not_depend_on_other_requests():
    b = Batch(11, "bf16", 8, 2, 128, posts([50, 9, 140]), 333)
    q, k, v, k2, v2 = b.device()
    whole = B.po_op_attention_shared(q, k, v, b.req, k2, v2, 333, q_prescaled=True)
    q[64:128] = NAN                                                       # another request's queries and keys
    k[64:128] = NAN
    v[:, 64:128] = NAN
    again = B.po_op_attention_shared(q, k, v, b.req, k2, v2, 333, q_prescaled=True)
    assert torch.equal(whole[:50], again[:50]) and torch.equal(whole[128:268], again[128:268])
    assert bool(torch.isnan(again[64:73].float()).all())


def test_own_keys_beyond_32_bits():
    """rows of k and columns of V^T whose byte offsets pass 2^32"""
    rows = (1 << 21) + 4096                                               # x 2 heads x 512 elements x 2 bytes
    far = [(0, 3, rows - 200, 150), (3, 70, rows - 800, 70)]
    hq, hkv, hd, n2 = 16, 8, 128, 100
    b = Batch(12, "bf16", hq, hkv, hd, [(0, 3, 0, 150), (3, 70, 152, 70)], n2)
    q, k, v, k2, v2 = b.device()
    kf = torch.empty(rows, hkv, hd, dtype=torch.bfloat16, device="cuda")
    vf = torch.empty(hkv * hd, rows, dtype=torch.bfloat16, device="cuda")
    for (_, _, a, n), (_, _, t, _) in zip(b.req.tolist(), far):
        kf[t:t + n] = k[a:a + n]
        vf[:, t:t + n] = v[:, a:a + n]
    want = B.po_op_attention_shared(q, k, v, b.req, k2, v2, n2, q_prescaled=True)
    got = B.po_op_attention_shared(q, kf, vf, far, k2, v2, n2, q_prescaled=True)
    assert torch.equal(got, want)


def test_captured_and_replayed_on_another_stream():
    cases = [Batch(13, "bf16", 8, 2, 128, posts([50, 9, 140]), 900), Batch(14, "bf16", 8, 2, 128, singles([50, 9, 140]), 900)]
    ins = [b.device() for b in cases]

    def both():
        return [B.po_op_attention_shared(t[0], t[1], t[2], b.req.copy(), t[3], t[4], b.n2, q_prescaled=True) for b, t in zip(cases, ins)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for i in range(3):
        for t in ins:
            t[0].copy_(torch.randn(t[0].shape, device="cuda"))
        want = both()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_binding_refuses_what_the_library_cannot_see():
    b = Batch(15, "bf16", 8, 2, 128, posts([50, 9]), 100)
    q, k, v, k2, v2 = b.device()
    f = B.po_op_attention_shared
    for args, kw in (((q, k.float(), v, b.req), {}), ((q, k, v.t(), b.req), {}), ((q.cpu(), k, v, b.req), {}),
                     ((q, k, v, b.req), {"k2": k2, "v2": v2, "n2": k2.shape[0] + 1}), ((q, k, v, b.req), {"n2": 10}),
                     ((q, k, v, b.req[:, :3]), {}), ((q[:, :, :64].contiguous(), k, v, b.req), {})):
        with pytest.raises(ValueError):
            f(*args, **kw)
    for bad in ([(0, q.shape[0] + 1, 0, 5)], [(0, 5, 0, k.shape[0] + 1)], [(5, 5, 0, 5), (0, 5, 8, 5)], [(0, 5, 0, 5), (4, 5, 8, 5)], [(0, 5, 4, 5)], [(0, -1, 0, 5)], [(-1, 5, 0, 5)], np.zeros((0, 4))):
        with pytest.raises(B.PoError):
            f(q, k, v, np.array(bad, dtype=np.int64).reshape(-1, 4))
