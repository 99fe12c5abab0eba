"""The drawing kernels run on the CPU (tests/sample_on_cpu.py), with each wavefront as far ahead of the others as the barriers allow:
all threads have to meet at the same barriers and the tokens have to be the definition's, in whatever order wavefronts run.
Oracle and tolerances: tests/test_gpu_sample.py."""
import numpy as np
import pytest

import sample_on_cpu as S
from test_gpu_sample import draw64


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return S.build(str(tmp_path_factory.mktemp("sample")))


def check(lib, z, u, t=None, k=None, p=None, mp=None, order="ascending"):
    tok, lp = S.sample(lib, z, u, t, k, p, mp, order)
    f32 = np.float32
    for i in range(len(z)):
        at = lambda a, default, ty: default if a is None else ty(a[i])
        want, wl = draw64(z[i].copy(), f32(u[i]), at(t, f32(1), f32), at(k, 0, int), at(p, f32(1), f32), at(mp, f32(0), f32))
        assert tok[i] == want, (i, tok[i], want)
        assert lp[i] == wl or abs(lp[i] - wl) <= 2.0 ** -24 * abs(wl) + 2e-11, (i, lp[i], wl)


orders = pytest.mark.parametrize("order", S.ORDERS)


@orders
def test_every_kind_of_row(lib, order):
    rng = np.random.default_rng(1)
    z = (rng.standard_normal((8, 5000)) * 2).astype(np.float32)
    z[::2] = np.round(z[::2] * 8) / 8
    check(lib, z, rng.random(8, dtype=np.float32), [1.0, 0.8, 0.5, 0.0, 1.0, 1.0, 1.0, 2.0], [0, 50, 0, 0, 3000, 3000, 0, 0],
          [0.9, 0.9, 0.7, 1.0, 0.8, 1.0, 1.0, 1.0], [0.0, 0.0, 0.1, 0.0, 0.0, 0.01, 0.1, 0.0], order)


@orders
def test_more_equal_logits_than_a_list_holds(lib, order):
    """top_k beyond what parts list, and a bin of thousands of tokens: the whole row is searched, twice with top_p"""
    rng = np.random.default_rng(2)
    z = np.zeros((4, 20011), dtype=np.float32)
    z[2:] = (rng.standard_normal((2, 20011)) * 0.5).astype(np.float32)
    z[2:, ::3] = 0.25
    check(lib, z, rng.random(4, dtype=np.float32), None, [9000, 0, 12000, 0], [1.0, 0.5, 0.7, 0.6], None, order)


@orders
def test_parts_whose_lists_together_are_longer_than_one(lib, order):
    """five parts of about 1800 equal largest logits each"""
    rng = np.random.default_rng(3)
    z = (rng.standard_normal((2, 70000)) * 0.5).astype(np.float32)
    z[:, ::9] = 3.0
    check(lib, z, rng.random(2, dtype=np.float32), None, [900, 900], [1.0, 0.5], None, order)


@pytest.mark.parametrize("p,k", [(0.37, None), (0.71, 1600000)])
def test_millions_of_equal_logits(lib, p, k):
    """their weights all fall into one bin of whole numbers"""
    z = np.full((1, (1 << 21) + 77), 0.5, dtype=np.float32)
    check(lib, z, [0.83], None, k and [k], [p])
