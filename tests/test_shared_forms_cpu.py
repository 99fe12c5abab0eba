"""How attention behind a shared prefix is divided, and what that asks of the scratch (no GPU)."""
import ctypes as C

import numpy as np
import pytest

from paper_2505_07203_amd import binding as B
from tests.shared_forms import FORMS, SMALL, requests_of


@pytest.mark.parametrize("name", FORMS)
def test_the_form_of_a_batch(name):
    form, pieces, heads, spec, n2, given = FORMS[name]
    req = requests_of(spec)
    need = B.po_attention_shared_bytes(B.PO_BF16, req, n2, *heads)
    assert B.po_attention_shared_form(req, n2, *heads, need if given is None else given) == (form, pieces)
    if given is None:
        assert B.po_attention_shared_form(req, n2, *heads) == (form, pieces)          # (what is asked for is enough)


def test_every_form_is_among_them():
    assert {(f[0], f[1] > 1) for f in FORMS.values()} >= {("TOKENS", False), ("ROWS", False), ("TILES", False), ("TILES", True), ("SPLIT", False),
                                                         ("SPLIT", True), ("TILES_SPLIT", True), ("TILES_FINISH", True)}


def test_without_scratch_nothing_is_divided():
    for form, _, heads, spec, n2, _ in FORMS.values():
        got, pieces = B.po_attention_shared_form(requests_of(spec), n2, *heads, 0)
        assert got in ("TOKENS", "ROWS", "TILES") and pieces <= 1


def test_requests_without_a_row():
    assert B.po_attention_shared_form([(0, 0, 0, 0)], 500, *SMALL) == ("TOKENS", 0)
    assert B.po_attention_shared_bytes(B.PO_BF16, [(0, 0, 0, 0)], 500, *SMALL) == 0


def test_refusals():
    req = np.array([(0, 1, 0, 5)], dtype=np.int64)
    f, p = C.c_int32(0), C.c_int32(0)
    ask = lambda r=req.ctypes.data, n=1, n2=100, hq=32, hkv=8, hd=128, a=C.byref(f), b=C.byref(p): B.lib().po_attention_shared_form(
        r, n, n2, hq, hkv, hd, 1 << 30, a, b)
    assert ask() == B.PO_OK
    for kw in (dict(r=None), dict(n=0), dict(n2=-1), dict(hq=31), dict(hkv=0), dict(a=None), dict(b=None)):
        assert ask(**kw) == B.PO_ERR_INVALID_ARG, kw
    assert ask(hd=96) == B.PO_ERR_BAD_CONFIG
    assert ask(n2=(1 << 24) + 1) == B.PO_ERR_TOO_LONG
    for rows in ([(0, 1 << 24, 0, 0)], [(i << 19, 1 << 19, 0, 0) for i in range(128)]):           # more rows and heads than 32 bits count
        many = np.array(rows, dtype=np.int64)
        assert ask(r=many.ctypes.data, n=len(many), hq=4096, hkv=1, hd=64) == B.PO_ERR_TOO_LONG
    long = np.array([(0, 1 << 20, 0, 1 << 24)], dtype=np.int64)                                  # ... and more pieces than a launch has
    assert ask(r=long.ctypes.data, hq=32, hkv=8, n2=0) == B.PO_OK and B.SHARED_FORMS[f.value] in ("TOKENS", "ROWS")
    bad = np.array([(0, 2, 0, 5), (1, 1, 0, 5)], dtype=np.int64)                       # rows of q that meet
    assert ask(r=bad.ctypes.data, n=2) == B.PO_ERR_INVALID_ARG
