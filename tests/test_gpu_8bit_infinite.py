"""Weight gradients of activations in E5M2 that are infinite."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.eight_bit import values
from tests.test_gpu_8bit_weight_grad import AG, inputs, run

pytestmark = pytest.mark.gpu


def test_infinite_activations_stay_infinite():
    """E5M2 has infinities, which the products and the way back keep; G's finite numbers, of one sign, take them through.  Next to them NaN,
    and numbers as they were."""
    P, M, N, K = 1, 70, 16, 272
    d, x = inputs(AG, P, M, N, K, api.DTYPE_E5M2, 60, whole=True)
    d = [t.abs() + 1 for t in d]
    clean = run(AG, P, M, N, K, api.DTYPE_E5M2, d, x, api.DTYPE_FP32)[0]
    x[0][0].view(torch.uint8)[3, 5], x[0][0].view(torch.uint8)[69, 130], x[0][0].view(torch.uint8)[64, 271] = 0x7C, 0xFC, 0x7E
    got = run(AG, P, M, N, K, api.DTYPE_E5M2, d, x, api.DTYPE_FP32)[0]
    assert (got[:, 5] == float("inf")).all() and (got[:, 130] == float("-inf")).all() and got[:, 271].isnan().all()
    rest = [c for c in range(K) if c not in (5, 130, 271)]
    assert torch.equal(got[:, rest], clean[:, rest])
    # against one another, and against a zero: no number
    x[0][0].view(torch.uint8)[4, 5] = 0xFC
    d[0][69, 3] = 0
    got = run(AG, P, M, N, K, api.DTYPE_E5M2, d, x, api.DTYPE_FP32)[0]
    assert got[:, 5].isnan().all() and got[3, 130].isnan() and (got[:3, 130] == float("-inf")).all()


@pytest.mark.parametrize("first", [0, 1, 100, 127, 200, 247, 254])
def test_every_number_beside_an_infinite_one(first):
    """One row each, every number of E5M2 with every scale of a few: as BF16 holds them, infinities and NaN too."""
    bits = torch.arange(256, device="cuda", dtype=torch.uint8).view(1, 256)
    scales = torch.tensor([[first, min(254, first + 7)]], dtype=torch.uint8, device="cuda")
    x = bits.view(torch.float8_e5m2), scales.view(torch.float8_e8m0fnu)
    got = run(AG, 1, 1, 8, 256, api.DTYPE_E5M2, [torch.ones(1, 8, device="cuda", dtype=torch.bfloat16)], [x], api.DTYPE_FP32)[0]
    want = values(*x).float().bfloat16().float().expand(8, 256)
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(nan=0.0, posinf=3e38, neginf=-3e38), want.nan_to_num(nan=0.0, posinf=3e38, neginf=-3e38))
