"""Drawing tokens from rows of millions of logits, where each of the many has 10^-7 of the weight or less: a sum that is off by 10^-6 of
the whole ends top_p at another token and moves draws by one.  Oracle and tolerances: tests/test_gpu_sample.py."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def far_above_the_bulk(seed, V, rows):
    z = np.random.default_rng(seed).standard_normal((rows, V)).astype(np.float32)
    z[:, V // 3] = 14.0
    return z


@pytest.mark.parametrize("V,rows", [(1 << 22, 3), ((1 << 23) + 1001, 2), (1 << 24, 1)])
def test_weights_far_below_the_largest_count_in_full(V, rows):
    z, u = far_above_the_bulk(V, V, rows), [0.93, 0.31, 0.62][:rows]
    check(z, u, None, None, [0.9] * rows)
    check(z, u)


def test_weights_far_below_the_largest_with_top_k():
    z = far_above_the_bulk(3, 1 << 22, 3)
    z[:2, 1::2] = np.round(z[:2, 1::2] * 2) / 2
    check(z, [0.29, 0.71, 0.87], None, [3000000, 1500000, 2500000], [0.8, 1.0, 0.97])


def test_millions_of_equal_logits():
    z = np.full((3, (1 << 22) + 77), 0.5, dtype=np.float32)
    z[2, ::3] = 0.25
    check(z, [0.83, 0.4, 0.6], None, [0, 3000001, 0], [0.37, 0.71, 0.93])


def test_vocabularies_of_the_bf16_grid():
    """thousands of tokens to a value, a large one above them; top_p near 1"""
    rng = np.random.default_rng(5)
    z = torch.from_numpy((rng.standard_normal((8, 128256)) + 10).astype(np.float32)).to(torch.bfloat16).float().numpy()
    z[:, 77] = 26.0
    check(z, rng.random(8, dtype=np.float32), None, [0, 0, 0, 0, 20000, 90000, 900, 0], [0.999, 0.9995, 0.9999, 0.99995, 0.99, 0.9995, 0.9, 0.99999])


def test_signalling_nans():
    """as memory that nobody wrote may hold them; and rows of random bits"""
    rng = np.random.default_rng(9)
    z = (rng.standard_normal((6, 20000)) * 2).astype(np.float32)
    z[:, 100], z[:, 17100] = 12.0, 11.5
    bits = z.view(np.uint32)
    bits[:, 164], bits[:, 17164], bits[:, 17228] = 0x7fa00000, 0xffa00000, 0x7f800001
    bits[3, 200:9000] = 0x7fbfffff
    with np.errstate(all="ignore"):
        check(z, rng.random(6, dtype=np.float32), [1.0, 1.0, 0.0, 0.7, 1.0, 1.0], [0, 50, 0, 0, 0, 3000], [1.0, 0.9, 1.0, 0.9, 1.0, 0.8],
              [0.0, 0.0, 0.0, 0.0, 0.1, 0.0])
        check(z, rng.random(6, dtype=np.float32))
        for V in (1, 70, 4000, 40000, 70000):
            for k in (None, [1, 20, 1000, 1025, 3000, 0, 5, 60] * 4):
                check(rng.integers(0, 2 ** 32, (32, V), dtype=np.uint32).view(np.float32), rng.random(32, dtype=np.float32), [0.5, 1.0, 100.0, 1e30] * 8, k,
                      k and [0.9, 0.5] * 16)
