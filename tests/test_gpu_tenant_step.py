"""A step of many tenants' requests as a program would run it: residual, norm and codes in one call; the shared FP8 product beside the tenants'
adapters, which read the same call's bf16 rows; the next norm; the prompt scored through the LM head, and the requests' last rows as logits
with their alternatives.  Every operator's result is compared with float64 arithmetic on the inputs it was given (tolerances as in its own
tests), the whole in a graph, replayed between other work, with the eager run, and two steps at once on two streams with each alone."""
import numpy as np
import pytest
import torch

from paper_2505_07203_amd import binding as B
from tests.test_gpu_adapters import reference
from tests.test_gpu_fp8_block_tiles import sum_err, values
from tests.test_gpu_head_logprobs import check as check_head
from tests.test_gpu_logprobs import check as check_logits
from tests.test_gpu_norm_quant import check as check_norm

pytestmark = pytest.mark.gpu

D, V = 512, 9001
LENS = [33, 1, 70, 128, 5, 1]
ADAPTER = [2, 0, -1, 1, 0, 2]
RANKS, SCALES = [16, 64, 5], [0.5, 0.25, 2.0]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class Step:
    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s, scale=1.0: (torch.randn(*s, device="cuda", generator=g) * scale).to(torch.bfloat16)
        rows = sum(LENS)
        self.x, self.delta = rnd(rows, D), rnd(rows, D, scale=0.3)
        self.g1, self.g2 = (rnd(D, scale=0.1) + 1 for _ in range(2))
        self.w = B.po_op_quantize_blocks(rnd(D, D, scale=0.03), 128)
        self.a, self.b = rnd(3, 64, D, scale=0.04), rnd(3, D, 64, scale=0.1)
        self.head = rnd(V, D, scale=0.05)
        self.next = torch.randint(0, V, (rows,), device="cuda", generator=g).to(torch.int32)
        first = np.cumsum([0] + LENS)
        self.seg = np.array([(first[i], LENS[i], ADAPTER[i]) for i in range(len(LENS))], dtype=np.int64)
        self.last = torch.from_numpy(first[1:] - 1).cuda()

    def run(self):
        r = {}
        r["h"], r["codes"], r["scales"], r["y"] = B.po_op_add_rmsnorm_quantize(self.x, self.delta, self.g1, 1e-5, block=128, normed=True)
        r["p"] = B.po_op_linear_fp8_block(r["codes"], r["scales"], *self.w, residual=r["h"])
        r["o"] = B.po_op_adapters(r["y"], self.a, self.b, RANKS, SCALES, self.seg, residual=r["p"])
        _, _, _, r["n"] = B.po_op_add_rmsnorm_quantize(r["o"], None, self.g2, 1e-5, normed=True, codes=False)
        r["lp"], r["ent"] = B.po_op_lm_head_logprobs(r["n"], self.head, self.next)
        r["z"] = torch.stack([B.po_op_lm_head(x, self.head) for x in r["n"][self.last]])
        r["glp"], r["gent"], r["ids"], r["tlp"] = B.po_op_token_logprobs(r["z"], self.next[self.last][:, None].contiguous(), top=7)
        return r


NAMES = ("h", "codes", "scales", "y", "p", "o", "n", "lp", "ent", "glp", "gent", "ids", "tlp")


def test_every_result_by_its_definition():
    s = Step(1)
    r = s.run()
    check_norm(s.x, s.delta, s.g1, 128, 1e-5, r["h"], r["codes"], r["scales"], r["y"])
    av, wv = values(r["codes"], r["scales"], 1), values(*s.w, 128)
    want, e = av @ wv.t() + r["h"].double(), sum_err(av, wv)
    assert bool(((r["p"].double() - want).abs() <= 2.0 ** -8 * (want.abs() + e) + e + 1e-30).all())
    want, e = reference(r["y"], s.a, s.b, RANKS, SCALES, s.seg.tolist(), r["p"])
    assert bool(((r["o"].double() - want).abs() <= 2.0 ** -8 * (want.abs() + e) + e).all())
    check_norm(r["o"], None, s.g2, 128, 1e-5, r["o"], None, None, r["n"])
    check_head(r["n"], s.head, s.next, r["lp"], r["ent"])
    check_logits(r["z"], s.next[s.last][:, None].contiguous(), 7)
    # the two ways to a log-probability: float32 sums of 512 products in two orders, 2 * 512 roundings of 2^-24 of their terms' sum
    off = 2 * (512 * 2.0 ** -24 * (r["n"][s.last].double().abs() @ s.head.double().abs().t()).amax(1) + 2.0 ** -24 * 256)
    assert bool(((r["lp"][s.last] - r["glp"][:, 0]).double().abs() <= off).all())


def test_captured_whole():
    s = Step(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = s.run()
    other = Step(3)
    for seed in range(3):
        torch.manual_seed(seed)
        s.x.copy_(torch.randn(s.x.shape, device="cuda").to(torch.bfloat16))
        s.a.copy_(torch.randn(s.a.shape, device="cuda").to(torch.bfloat16) * 0.05)
        want = s.run()
        other.run()
        g.replay()
        torch.cuda.synchronize()
        for name in NAMES:
            assert torch.equal(got[name], want[name]), name


def test_two_streams_at_once():
    """each call allocates scratch of its own, on its stream"""
    steps = [Step(4), Step(5)]
    want = [s.run() for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(4):
        got = []
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                got.append(s.run())
        torch.cuda.synchronize()
        for w, o in zip(want, got):
            assert all(torch.equal(w[n], o[n]) for n in NAMES)
