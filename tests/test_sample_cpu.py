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


def far_above_the_bulk(rng, V, top=14.0):
    """one token that holds much of the weight, the rest spread over millions, 10^-7 of the whole or less each"""
    z = rng.standard_normal((1, V)).astype(np.float32)
    z[0, V // 3] = top
    return z


@pytest.mark.parametrize("seed", [1, 2])
def test_weights_far_below_the_largest_count_in_full(lib, seed):
    z = far_above_the_bulk(np.random.default_rng(seed), 1 << 22)
    for u in (0.31, 0.62, 0.93):
        check(lib, z, [u], None, None, [0.9])


def test_weights_far_below_the_largest_with_top_k(lib):
    rng = np.random.default_rng(3)
    z = far_above_the_bulk(rng, 1 << 21)
    z[0, 1::2] = np.round(z[0, 1::2] * 2) / 2
    for u in (0.29, 0.71):
        check(lib, z, [u], None, [1500000], [0.8])


@pytest.mark.parametrize("T", [1.0, 0.05, 0.01, 0.001])
@pytest.mark.parametrize("k", [0, 900, 45000])
def test_plateaus_far_below_the_largest(lib, T, k):
    """60000 tokens of three values, 21 to 22 powers of e below one: keys with the same leading bits, and weights hundreds of powers apart at
    the low temperatures.  top_p ends in the middle of what top_k leaves; u near 1, since the one token has all but 10^-5 of the weight"""
    z = np.resize(np.array([69.0 + 3 * T, 69.0 + 2.5 * T, 69.0 + 2 * T], dtype=np.float32), (1, 60000))
    z[0, 7] = 69.0 + 24 * T
    w = np.sort(np.exp((z[0].astype(np.float64) - z[0].max()) / np.float64(np.float32(T))))[::-1][:k or None]
    c = np.cumsum(w)

    def away_from_the_sums(x, sums):
        """the next lower number that no running sum is near to: the weights are 7e-10 of the whole and less"""
        x = np.float32(x)
        while np.abs(sums - np.float64(x) * sums[-1]).min() < 5e-11 * sums[-1]:
            x = np.nextafter(x, np.float32(0))
        return x
    p = away_from_the_sums(c[len(c) // 2] / c[-1], c)
    assert p < 1 and c[0] < np.float64(p) * c[-1]
    n = 1 + int(np.searchsorted(c, np.float64(p) * c[-1]))
    w = np.exp((z[0].astype(np.float64) - z[0].max()) / np.float64(np.float32(T)))
    kept = np.cumsum(w[np.sort(np.argsort(-z[0], kind="stable")[:n])])
    for u in (0.2, 1 - 2.0 ** -18, 1 - 2.0 ** -24):
        check(lib, z, [away_from_the_sums(u, kept)], [T], [k] if k else None, [p])


def test_bulk_that_shares_a_bin_with_a_far_larger_token(lib):
    """two million equal weights, 10 powers of e below the largest and in one bin of leading bits with it, each half a digit off there; the last
    kept token is among 3000 neighbouring numbers in the next bin, at the end of the row"""
    T, V, n = np.float32(0.18), 1 << 21, 3000
    top = np.float32(13.9)
    near = np.float32(12.1) + np.arange(4000, dtype=np.float32) * np.float32(2.0 ** -20)
    digits = np.exp((near.astype(np.float64) - np.float64(top)) / np.float64(T)) * 2.0 ** 40
    z = np.full((1, V), near[np.argmin(np.abs(digits - np.floor(digits) - 0.5))], dtype=np.float32)
    z[0, 5], z[0, 9] = top, -20.0
    z[0, -n:] = np.float32(11.2) - np.arange(n, dtype=np.float32) * np.float32(2.0 ** -20)
    w = np.exp((z[0].astype(np.float64) - np.float64(top)) / np.float64(T))
    c = np.cumsum(np.sort(w)[::-1])
    for share in (c[-n // 2], c[-n // 3]):
        check(lib, z, [1 - 2.0 ** -24], [T], None, [share / c[-1]])


def test_signalling_nans(lib):
    """as memory that nobody wrote may hold them, each behind a larger logit that the same thread reads: of the two the number counts"""
    rng = np.random.default_rng(9)
    z = (rng.standard_normal((6, 20000)) * 2).astype(np.float32)
    z[:, 100], z[:, 17100] = 12.0, 11.5
    bits = z.view(np.uint32)
    bits[:, 164], bits[:, 17164], bits[:, 17228] = 0x7fa00000, 0xffa00000, 0x7f800001
    bits[3, 200:9000] = 0x7fbfffff
    with np.errstate(invalid="ignore"):
        check(lib, z, rng.random(6, dtype=np.float32), [1.0, 1.0, 0.0, 0.7, 1.0, 1.0], [0, 50, 0, 0, 0, 3000], [1.0, 0.9, 1.0, 0.9, 1.0, 0.8],
              [0.0, 0.0, 0.0, 0.0, 0.1, 0.0])
        check(lib, z, rng.random(6, dtype=np.float32))
