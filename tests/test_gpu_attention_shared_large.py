"""Attention behind a shared prefix where scores are so large that float32 holds them to whole powers of 2 only, up to what the
interface allows: results stay finite and inside what the values span, in every form and for queries with and without their factor."""
import math

import numpy as np
import pytest
import torch

from paper_2505_07203_amd import binding as B
from tests.shared_forms import FORMS, requests_of
from tests.test_gpu_attention_shared import Batch
from tests.test_gpu_attention_shared_forms import compare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pre", [True, False])
@pytest.mark.parametrize("name", FORMS)
def test_scores_up_to_2_to_29(name, pre):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    form, pieces, (hq, hkv, hd), spec, n2, given = FORMS[name]
    req = np.array(requests_of(spec), dtype=np.int64).reshape(-1, 4)
    g = torch.Generator(device="cuda")
    g.manual_seed(len(name))
    rows, keys, n2c = (int(x + 7) // 8 * 8 for x in ((req[:, 0] + req[:, 1]).max(), max((req[:, 2] + req[:, 3]).max(), 1), max(n2, 1)))
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
    # queries are 2^14 along the first dimension and 0 otherwise, so that a key's first value alone makes its score: 2^29 at most
    factor = 1.0 if pre else B.attention_q_scale(hd)
    q = torch.zeros(rows, hq, hd, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 2.0 ** 14
    most = 2.0 ** 15 / 2.0 ** math.ceil(math.log2(factor))
    spread = lambda n: ((torch.rand(n, hkv, generator=g, device="cuda") * 2 - 1) * most).to(torch.bfloat16)
    k, k2, v, v2 = rnd(keys, hkv, hd), rnd(n2c, hkv, hd), rnd(hkv * hd, keys), rnd(hkv * hd, n2c)
    k[..., 0], k2[..., 0] = spread(keys), spread(n2c)
    size = B.po_attention_shared_bytes(B.PO_BF16, req, n2, hq, hkv, hd) if given is None else given
    o = B.po_op_attention_shared(q, k, v, req, k2, v2, n2, q_prescaled=pre, scratch=torch.empty(size, dtype=torch.uint8, device="cuda"))
    top = float(torch.maximum(v.abs().max(), v2.abs().max()))
    assert float(o.float().abs().max()) <= top * (1 + 2.0 ** -8)             # (NaN fails this too)
    for q0, nq, k0, nk in req.tolist():
        if nq and n2 + nk > 0 and n2:
            assert bool((o[q0:q0 + nq].float().abs().amax((1, 2)) > 0).all())


@pytest.mark.parametrize("above", [0.0, 14.5, -14.5])
@pytest.mark.parametrize("name", FORMS)
def test_values_up_to_2_to_63(name, above):
    """the same, with own keys' scores 29 powers of 2 above the prefix's or below them: definition and tolerances of
    tests/test_gpu_attention_shared.py, which go with the values"""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    form, pieces, (hq, hkv, hd), spec, n2, given = FORMS[name]
    if n2 * sum(s[0] * s[1] for s in spec) > 2e6:
        pytest.skip("a long reference")
    b = Batch(len(name), "bf16", hq, hkv, hd, requests_of(spec), n2)
    b.q[..., 0] = 2.0
    b.k[..., 0] = torch.where(b.k[..., 0].isnan(), b.k[..., 0], torch.full_like(b.k[..., 0], above))
    b.k2[:n2, :, 0] = 0.0
    b.v, b.v2 = b.v * 2.0 ** 60, b.v2 * 2.0 ** 60                            # (of a few times 1 each)
    q, k, v, k2, v2 = b.device()
    out = torch.full_like(q, 777.0)
    mark = out.clone()
    size = B.po_attention_shared_bytes(B.PO_BF16, b.req, n2, hq, hkv, hd) if given is None else given
    B.po_op_attention_shared(q, k, v, b.req, k2, v2, n2, out=out, q_prescaled=b.pre, scratch=torch.empty(size, dtype=torch.uint8, device="cuda"))
    compare(b, out, mark)
