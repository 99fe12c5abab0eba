"""Every way in which attention behind a shared prefix is divided among workgroups, at ragged sizes: the same definition and tolerances
as tests/test_gpu_attention_shared.py, and that the way asked for is the one that runs."""
import pytest
import torch

from paper_2505_07203_amd import binding as B
from tests.shared_forms import FORMS, WIDE_F32, requests_of
from tests.test_gpu_attention_shared import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def compare(b, got, mark):
    want, tol = b.reference()
    asked = ~torch.isnan(want[:, 0, 0])
    d = (got.cpu().double() - want).abs()[asked]
    assert (d <= tol[asked]).all(), (int((~(d <= tol[asked])).sum()), float((d / tol[asked]).max()))
    assert torch.equal(got.cpu()[~asked], mark.cpu()[~asked])


@pytest.mark.parametrize("name", FORMS)
def test_a_form(name):
    form, pieces, heads, spec, n2, given = FORMS[name]
    hq, hkv, hd = heads
    b = Batch(len(name), "bf16", hq, hkv, hd, requests_of(spec), n2)
    need = B.po_attention_shared_bytes(B.PO_BF16, b.req, n2, hq, hkv, hd)
    size = need if given is None else given
    assert B.po_attention_shared_form(b.req, n2, hq, hkv, hd, size) == (form, pieces)
    q, k, v, k2, v2 = b.device()
    scratch = torch.full((size + 64,), 0xff, dtype=torch.uint8, device="cuda")            # (NaN as float32)
    for in_place in (False, True):
        out = q if in_place else torch.full_like(q, 777.0)
        mark = out.clone()
        B.po_op_attention_shared(q, k, v, b.req, k2, v2, n2, out=out, q_prescaled=b.pre, scratch=scratch[:size])
        compare(b, out, mark)
    assert bool((scratch[size:] == 0xff).all())                                           # (nothing behind it)


@pytest.mark.parametrize("name", WIDE_F32)
def test_float32_with_128_rows_a_workgroup(name):
    (hq, hkv, hd), spec, n2 = WIDE_F32[name]
    b = Batch(len(name), "f32", hq, hkv, hd, requests_of(spec), n2)
    q, k, v, k2, v2 = b.device()
    for in_place in (False, True):
        out = q if in_place else torch.full_like(q, 777.0)
        mark = out.clone()
        B.po_op_attention_shared(q, k, v, b.req, k2, v2, n2, out=out)
        compare(b, out, mark)


@pytest.mark.parametrize("name", FORMS)
def test_a_request_with_nan_keys_and_values_spoils_no_other(name):
    form, pieces, (hq, hkv, hd), spec, n2, given = FORMS[name]
    b = Batch(len(name), "bf16", hq, hkv, hd, requests_of(spec), n2)
    q, k, v, k2, v2 = b.device()
    size = B.po_attention_shared_bytes(B.PO_BF16, b.req, n2, hq, hkv, hd) if given is None else given
    run = lambda: B.po_op_attention_shared(q, k, v, b.req, k2, v2, n2, q_prescaled=b.pre, scratch=torch.empty(size, dtype=torch.uint8, device="cuda"))
    want = run()
    with_keys = [r for r in b.req.tolist() if r[1] > 0 and r[3] > 0]
    for q0, nq, k0, nk in (with_keys[0], with_keys[len(with_keys) // 2], with_keys[-1]):
        keep = k[k0:k0 + nk].clone(), v[:, k0:k0 + nk].clone()
        k[k0:k0 + nk], v[:, k0:k0 + nk] = float("nan"), float("inf")
        got = run()
        k[k0:k0 + nk], v[:, k0:k0 + nk] = keep
        assert torch.equal(got[:q0], want[:q0]) and torch.equal(got[q0 + nq:], want[q0 + nq:])
        # queries of NaN too: a tile may then take the exponents' references of all its rows anew, so twice the tolerance of one result,
        # 2^-8 of the largest value for the probabilities' and the result's rounding each
        keep = q[q0:q0 + nq].clone()
        q[q0:q0 + nq] = float("nan")
        got = run()
        q[q0:q0 + nq] = keep
        got[q0:q0 + nq] = want[q0:q0 + nq]
        top = max(float(x.nan_to_num(0.0).abs().max()) for x in (b.v.float(), b.v2.float()))
        assert float((got.float() - want.float()).abs().max()) <= 4 * 2.0 ** -8 * top
        if len(with_keys) == 1:
            break


def test_scores_that_grow_along_the_keys():
    """the reference of the exponentials is left behind again and again, and by more than a float32 exponent covers"""
    for name in FORMS:
        form, pieces, (hq, hkv, hd), spec, n2, given = FORMS[name]
        if n2 * sum(s[0] * s[1] for s in spec) > 2e6:
            continue
        b = Batch(3, "bf16", hq, hkv, hd, requests_of(spec), n2)
        b.q[..., 0] = 2.0
        ramp = lambda n: (torch.arange(n).float() * (400.0 / max(n, 1)))[:, None].to(torch.bfloat16)
        b.k[..., 0] = torch.where(b.k[..., 0].isnan(), b.k[..., 0], ramp(b.k.shape[0]).expand(-1, hkv) + 300)
        b.k2[:n2, :, 0] = ramp(n2)
        q, k, v, k2, v2 = b.device()
        out = torch.full_like(q, 777.0)
        mark = out.clone()
        B.po_op_attention_shared(q, k, v, b.req, k2, v2, n2, out=out, q_prescaled=b.pre)
        compare(b, out, mark)


def test_one_scratch_for_two_captured_calls():
    """two graphs over the same scratch, replayed in turn on one stream: every replay writes what it reads"""
    form, pieces, (hq, hkv, hd), spec, n2, _ = FORMS["finish"]
    a, b = (Batch(s, "bf16", hq, hkv, hd, requests_of(spec), n2) for s in (1, 2))
    size = B.po_attention_shared_bytes(B.PO_BF16, a.req, n2, hq, hkv, hd)
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    graphs = []
    for x in (a, b):
        q, k, v, k2, v2 = x.device()
        out = torch.zeros_like(q)
        run = lambda o: B.po_op_attention_shared(q, k, v, x.req, k2, v2, n2, out=o, q_prescaled=x.pre, scratch=scratch)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = run(torch.zeros_like(q))
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(out)
        graphs.append((g, out, want, (q, k, v, k2, v2)))
    for i in range(4):
        g, out, want, _ = graphs[i % 2]
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
