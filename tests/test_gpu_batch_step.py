"""One layer over a batch of requests behind a shared prefix and the draw of a token for each, as a program would run them: norm, QKV and
rotary embedding, attention behind the prefix, FP8 output product onto the residual, FP8 gate and up with SiLU, FP8 down onto the residual,
norm, head, draw.  Every operator's result is compared with float64 arithmetic on the inputs it was given (tolerances as in its own
tests), and the whole in a graph, replayed between other work, with the eager run, bit for bit."""
import math

import numpy as np
import pytest
import torch

from paper_2505_07203_amd import binding as B
from tests.test_gpu_fp8_block_tiles import sum_err, values
from tests.test_gpu_sample import draw64

pytestmark = pytest.mark.gpu

D, HQ, HKV, HD, F, V, N2 = 512, 8, 2, 128, 1408, 32001, 201
LENS = [33, 1, 70, 128, 5]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class Layer:
    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s, scale=1.0: (torch.randn(*s, device="cuda", generator=g) * scale).to(torch.bfloat16)
        self.prefix = rnd(N2, D)
        self.x = rnd(sum(LENS), D)
        self.g1, self.g2, self.g3 = (rnd(D, scale=0.1) + 1 for _ in range(3))
        self.wqkv, _ = B.po_op_pack_qkv(rnd(HQ * HD, D, scale=0.05), rnd(HKV * HD, D, scale=0.05), rnd(HKV * HD, D, scale=0.05), HQ, HKV, HD)
        self.wo = B.po_op_quantize_blocks(rnd(D, HQ * HD, scale=0.03), 128)
        (gate, sg), (up, su) = (B.po_op_quantize_blocks(rnd(F, D, scale=0.05), 128) for _ in range(2))
        self.gate, self.up = (gate, sg), (up, su)
        self.wgu = B.po_op_pack_gate_up(gate.view(torch.bfloat16), up.view(torch.bfloat16)).view(torch.uint8)
        self.sgu = torch.stack((sg, su))
        self.wd = B.po_op_quantize_blocks(rnd(D, F, scale=0.03), 128)
        self.head = rnd(V, D, scale=0.05)
        self.cos, self.sin = B.po_op_rope_table(N2 + max(LENS), HD, 5e5)
        n = len(LENS)
        self.u = torch.rand(n, device="cuda", generator=g)
        self.t = torch.tensor([0.7, 1.0, 0.0, 1.3, 0.9], device="cuda")
        self.k = torch.tensor([50, 0, 0, 1000, 5000], dtype=torch.int32, device="cuda")
        self.p = torch.tensor([0.95, 0.9, 1.0, 1.0, 0.8], device="cuda")
        # requests' own keys side by side, from multiples of 8 on
        self.first = np.cumsum([0] + LENS)
        self.at = np.cumsum([0] + [(n + 7) // 8 * 8 for n in LENS])
        self.req = [(int(self.first[i]), LENS[i], int(self.at[i]), LENS[i]) for i in range(n)]

    def run(self):
        r = {}
        scale = B.attention_q_scale(HD)
        qkv = lambda x, pos: B.po_op_qkv_rope(B.po_op_rmsnorm(x, self.g1, 1e-5), self.wqkv, None, self.cos, self.sin, HQ, HKV, HD, pos, q_scale=scale)
        _, k2, v2 = qkv(self.prefix, 0)
        q, k, v = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((len(self.x), HQ, HD), (int(self.at[-1]), HKV, HD), (HKV * HD, int(self.at[-1]))))
        for q0, n, k0, _ in self.req:
            qi, ki, vi = qkv(self.x[q0:q0 + n], N2)
            q[q0:q0 + n], k[k0:k0 + n], v[:, k0:k0 + n] = qi.view(n, HQ, HD), ki.view(n, HKV, HD), vi[:, N2:N2 + n]
        r["q"], r["k"], r["v"], r["k2"], r["v2"] = q, k, v, k2.view(N2, HKV, HD), v2
        r["o"] = B.po_op_attention_shared(q, k, v, self.req, r["k2"], v2, N2, q_prescaled=True)
        r["qo"] = B.po_op_quantize_blocks(r["o"].view(len(self.x), HQ * HD))
        r["h"] = B.po_op_linear_fp8_block(*r["qo"], *self.wo, residual=self.x)
        r["qn"] = B.po_op_quantize_blocks(B.po_op_rmsnorm(r["h"], self.g2, 1e-5))
        r["m"] = B.po_op_linear_fp8_block(*r["qn"], self.wgu, self.sgu, silu_mul=True)
        r["qm"] = B.po_op_quantize_blocks(r["m"])
        r["y"] = B.po_op_linear_fp8_block(*r["qm"], *self.wd, residual=r["h"])
        last = B.po_op_rmsnorm(torch.cat([r["y"][int(f) - 1:int(f)] for f in self.first[1:]]), self.g3, 1e-5)
        r["z"] = torch.stack([B.po_op_lm_head(x, self.head) for x in last])
        r["tok"], r["lp"] = B.po_op_sample(r["z"], self.u, self.t, self.k, self.p)
        return r


def test_every_result_by_its_definition():
    l = Layer(1)
    r = l.run()
    # attention: 2^-8 of a probability and of the result; the float32 terms (see its own tests) are below 2^-12 at these scores
    q, k, k2 = r["q"].double(), r["k"].double(), r["k2"].double()
    vt, v2t = r["v"].double(), r["v2"].double()
    for q0, n, k0, _ in l.req:
        hide = torch.arange(N2 + n, device="cuda")[None] > torch.arange(n, device="cuda")[:, None] + N2
        for h in range(HQ):
            c = h // (HQ // HKV)
            kk = torch.cat((k2[:, c], k[k0:k0 + n, c]))
            vv = torch.cat((v2t[c * HD:(c + 1) * HD, :N2].t(), vt[c * HD:(c + 1) * HD, k0:k0 + n].t()))
            s = (q[q0:q0 + n, h] @ kk.t() * math.log(2.0)).masked_fill(hide, -math.inf)
            assert float(s[~hide].abs().max()) < 100.0
            p = torch.softmax(s, 1)
            want, a = p @ vv, p @ vv.abs()
            got = r["o"][q0:q0 + n, h].double()
            assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * a * (1 + 2.0 ** -8)).all())

    def product(a, w, res, got):
        av, wv = values(*a, 1), values(*w, 128)
        want, e = av @ wv.t() + res.double(), sum_err(av, wv)
        assert bool(((got.double() - want).abs() <= 2.0 ** -8 * (want.abs() + e) + e + 1e-30).all())

    product(r["qo"], l.wo, l.x, r["h"])
    product(r["qm"], l.wd, r["h"], r["y"])
    av, gv, uv = values(*r["qn"], 1), values(*l.gate, 128), values(*l.up, 128)
    gate, up, eg, eu = av @ gv.t(), av @ uv.t(), sum_err(av, gv), sum_err(av, uv)
    want = gate / (1 + torch.exp(-gate)) * up
    e = 1.1 * eg * (up.abs() + eu) + gate.abs() * eu
    assert bool(((r["m"].double() - want).abs() <= 2.0 ** -8 * (want.abs() + e) + e + 2.0 ** -20 * want.abs() + 1e-30).all())
    z, u, t, kk, pp = (x.cpu().numpy() for x in (r["z"], l.u, l.t, l.k, l.p))
    for i in range(len(LENS)):
        tok, lp = draw64(z[i].copy(), u[i], t[i], kk[i], pp[i], np.float32(0.0))
        assert int(r["tok"][i]) == tok and abs(float(r["lp"][i]) - lp) <= 2.0 ** -24 * abs(lp) + 2e-11


def test_captured_whole():
    l = Layer(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        l.run()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = l.run()
    other = Layer(3)
    for seed in range(3):
        torch.manual_seed(seed)
        l.x.copy_(torch.randn(l.x.shape, device="cuda").to(torch.bfloat16))
        l.u.copy_(torch.rand(l.u.shape, device="cuda"))
        want = l.run()
        other.run()
        g.replay()
        torch.cuda.synchronize()
        for name in ("o", "h", "m", "y", "z", "tok", "lp"):
            assert torch.equal(got[name], want[name]), name
