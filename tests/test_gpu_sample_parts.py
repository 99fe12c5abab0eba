"""Drawing tokens where a row is cut into parts, its head is as long as a list, or its logits lie so close together that counting
by the leading bits of keys does not separate them.  Oracle and tolerances: tests/test_gpu_sample.py."""
import numpy as np
import pytest
import torch

from paper_2505_07203_amd import binding as B
from tests.test_gpu_sample import check, settings

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("rows,V", [(1, 128256), (1, 151937), (2, 262144), (3, 16384), (3, 16385), (5, 49153), (15, 65537), (17, 33000), (129, 32769), (300, 17001)])
def test_rows_of_several_parts(rows, V):
    rng = np.random.default_rng(V + rows)
    z = (rng.standard_normal((rows, V)) * rng.choice([0.2, 1.0, 3.0], (rows, 1))).astype(np.float32)
    z[::2] = torch.from_numpy(z[::2]).to(torch.bfloat16).float().numpy()
    check(z, rng.random(rows, dtype=np.float32), *settings(rng, rows))
    check(z[:3], rng.random(3, dtype=np.float32)[:rows], None, [40] * min(rows, 3))
    check(z[:3], rng.random(3, dtype=np.float32)[:rows], None, None, [0.9] * min(rows, 3))


def test_rows_longer_than_a_tile_of_1024_logits():
    """more than 2^20 logits: a tile is several reads long"""
    rng = np.random.default_rng(11)
    V = (1 << 20) + 4097
    z = (rng.standard_normal((4, V)) * 1.5).astype(np.float32)
    check(z, rng.random(4, dtype=np.float32))
    check(z, rng.random(4, dtype=np.float32), [0.9, 1.0, 0.7, 1.2], [0, 50, 3000, 0], [0.9, 0.8, 1.0, 1.0], [0.0, 0.0, 0.0, 0.2])


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 512, 513, 1023, 1024])
def test_a_head_of_n_tokens_far_above_the_rest(n):
    """a few logits high above a bulk that shares its keys' leading bits; top_k on both sides of n and of the longest that parts list"""
    rng = np.random.default_rng(n)
    V = 60000
    z = (rng.standard_normal((8, V)) * 0.4 - 30.9).astype(np.float32)
    for row in z:
        row[rng.permutation(V)[:n]] = np.linspace(0.0, 1.0, n, dtype=np.float32)
    k = [max(n - 1, 1), n, n + 1, 1024, 1025, 0, 0, min(n, 700)]
    check(z, rng.random(8, dtype=np.float32), [1.0, 0.7] * 4, k, [1.0, 0.9, 1.0, 1.0, 0.99, 0.9, 0.999999, 0.97])


def test_thousands_of_equal_logits_in_every_part():
    rng = np.random.default_rng(13)
    z = (rng.standard_normal((6, 70000)) * 0.5).astype(np.float32)
    z[:, ::2] = 3.0                                                              # 35000 equal ones at the top
    z[3:, 1::2] = 2.0
    check(z, rng.random(6, dtype=np.float32), None, [1, 900, 1024, 1025, 35000, 35001], [1.0, 0.5, 1.0, 0.7, 1.0, 0.9])
    check(z, rng.random(6, dtype=np.float32), None, None, [0.01, 0.5, 0.99, 0.25, 0.75, 0.999])


def test_parts_without_a_token():
    """all but one part masked; and only the last logit of the row left"""
    rng = np.random.default_rng(14)
    z = np.full((4, 100000), -np.inf, dtype=np.float32)
    z[0, 40000:40100] = rng.standard_normal(100)
    z[1, -1] = -4.0
    z[2, [0, 99999]] = 1.0
    for s in ((None,) * 4, ([1.0] * 4, [30] * 4, None, None), ([1.0] * 4, [2000] * 4, [0.9] * 4, None), ([1.0] * 4, None, [0.9] * 4, None),
              ([1.0] * 4, None, None, [0.3] * 4), ([0.0] * 4, None, None, None)):
        check(z, rng.random(4, dtype=np.float32), *s)


def test_what_an_earlier_call_left_in_the_scratch_does_not_show():
    rng = np.random.default_rng(15)
    scratch = torch.full((B.po_sample_bytes(9, 50000, True, True),), 0xff, dtype=torch.uint8, device="cuda")
    want = []
    for fresh in (True, False):
        for i in range(6):
            z = torch.from_numpy((np.random.default_rng(i).standard_normal((9, 50000)) * 2).astype(np.float32)).cuda()
            t, k, p, mp = (torch.from_numpy(np.asarray(a).astype(ty)).cuda()
                           for a, ty in zip(settings(np.random.default_rng(100 + i), 9), (np.float32, np.int32, np.float32, np.float32)))
            u = torch.from_numpy(np.random.default_rng(200 + i).random(9, dtype=np.float32)).cuda()
            tok, lp = B.po_op_sample(z, u, t, k, p, mp, **({} if fresh else {"scratch": scratch}))
            if fresh:
                want.append((tok, lp))
            else:
                assert torch.equal(tok, want[i][0]) and torch.equal(lp, want[i][1])


def test_one_row_or_one_column_of_any_pitch():
    rng = np.random.default_rng(16)
    z = torch.from_numpy((rng.standard_normal(5000) * 2).astype(np.float32)).cuda()
    u = torch.tensor([0.37], device="cuda")
    want = B.po_op_sample(z[None], u)
    for pitch in (1, 7, 4999):
        got = B.po_op_sample(z.as_strided((1, 5000), (pitch, 1)), u)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    tok, lp = B.po_op_sample(z.as_strided((3, 1), (7, 5)), u.repeat(3))
    assert tok.tolist() == [0, 0, 0] and lp.tolist() == [0.0, 0.0, 0.0]
