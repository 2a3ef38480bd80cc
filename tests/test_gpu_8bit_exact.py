"""Products of 8-bit operands whose sums FP32 holds exactly, at every shape: nothing but the rounding to BF16 is left, so a product that is
lost, doubled or taken from another row is seen wherever it is.  (Products are multiples of 2^-2 and at most 16; contractions are at most
32768 long: 19 bits before the point and 2 behind it.)"""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.test_gpu_8bit_products import AG, RS, SHAPES, exact, inputs, run

pytestmark = pytest.mark.gpu


def compare(op, P, M, N, K, layout, format, seed=70):
    a, b = inputs(op, P, M, N, K, layout, format, seed, whole=True)
    for o, e in zip(run(op, P, M, N, K, layout, format, a, b), exact(op, P, a, b, layout)):
        assert torch.equal(o, e.to(torch.bfloat16))


# clusters of the few-rows kernel: as many as run at once, and one more
@pytest.mark.parametrize("M", [1, 60, 130])
@pytest.mark.parametrize("tiles,K", [(15, 4096), (16, 4096), (33, 4096), (34, 4096), (45, 2048), (46, 4096), (70, 2064), (72, 2048), (93, 1040), (149, 1024), (200, 2048), (297, 528)])
def test_more_clusters_than_run_at_once(M, tiles, K):
    compare(AG, 1, M, 128 * tiles, K, api.B_NK, api.DTYPE_E4M3)
