"""The LM head's log-probabilities in every tile that its launches take, with one row tile and several, odd columns and ragged rows; and with weights of
256 MiB or more in one row tile, which are read past the caches.  Tolerances as in test_gpu_head_logprobs.  (rows, V, d); test_head_logprobs_tiles_cpu
holds that each list reaches every tile."""
import pytest
import torch

from paper_2505_07203_amd import binding as B
from test_gpu_head_logprobs import check, inputs

pytestmark = pytest.mark.gpu

BF16 = [(17, 34375, 512), (17, 309, 512), (69, 331, 192), (65, 17261, 320), (130, 10957, 320), (102, 17147, 512), (199, 10957, 320), (130, 16527, 512), (263, 10981, 512),
        (972, 10759, 512), (4099, 4097, 256), (130, 34329, 192), (129, 33001, 256), (259, 21825, 192), (19, 329, 128), (279, 323, 64), (193, 33001, 512), (194, 33931, 512), (395, 23099, 512)]
BF16_ONCE = [(1, 66001, 2048), (31, 66001, 2048), (50, 66001, 2048), (91, 66001, 2048), (128, 66001, 2048), (133, 66001, 2048), (187, 66001, 2048), (201, 66001, 2048), (150, 33001, 4096)]
F32 = [(1, 339, 100), (65, 307, 68), (31, 33001, 36), (1, 40000, 260), (11, 16521, 132), (17, 25067, 68), (17, 32001, 100), (33, 16387, 132), (65, 11051, 36), (130, 33000, 64), (49, 24585, 36), (49, 32001, 100), (104, 12489, 292)]
F32_ONCE = [(1, 17001, 4096), (17, 25067, 2680), (33, 17001, 4096), (49, 24585, 2736), (20, 8001, 8420)]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def run(rows, V, d, dtype):
    x, w, t = inputs(rows, V, d, rows + V + d, dtype)
    t[-1] = V - 1
    got = B.po_op_lm_head_logprobs(x, w, t)
    check(x, w, t, *got)
    x2 = x.clone()
    x2[rows // 2, 3] = float("nan")
    keep = torch.arange(rows, device="cuda") != rows // 2
    again = B.po_op_lm_head_logprobs(x2, w, t)                        # the same bits, whatever another row holds
    assert torch.equal(again[0][keep], got[0][keep]) and torch.equal(again[1][keep], got[1][keep])


@pytest.mark.parametrize("rows,V,d", BF16 + BF16_ONCE)
def test_bf16(rows, V, d):
    run(rows, V, d, torch.bfloat16)


@pytest.mark.parametrize("rows,V,d", F32 + F32_ONCE)
def test_float32(rows, V, d):
    run(rows, V, d, torch.float32)
