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


@pytest.mark.parametrize("op", [AG, RS])
@pytest.mark.parametrize("P,M,N,K", SHAPES)
def test_every_shape(op, P, M, N, K):
    compare(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3)


@pytest.mark.parametrize("op", [AG, RS])
@pytest.mark.parametrize("P,M,N,K", [s for s in SHAPES if s[2] % 16 == 0])
def test_every_shape_with_weights_along_n(op, P, M, N, K):
    compare(op, P, M, N, K, api.B_KN, api.DTYPE_E5M2)


# few tiles of a long contraction: rows in pieces, several shards a tile and a last tile of fewer, boundaries of ranks inside a tile,
# ranks' slices that end inside a scale's block
@pytest.mark.parametrize("layout", [api.B_NK, api.B_KN])
@pytest.mark.parametrize("op,P,M,N,K", [
    (AG, 1, 257, 80, 4112), (AG, 2, 1202, 112, 8192), (AG, 16, 640, 64, 4112), (AG, 16, 1600, 80, 6160), (AG, 5, 95, 16, 16400),
    (RS, 8, 600, 112, 2064), (RS, 3, 807, 48, 4096), (RS, 16, 4112, 16, 2048), (RS, 8, 152, 96, 3120), (RS, 16, 16, 64, 1168), (AG, 1, 1, 48, 32768),
])
def test_row_tiles(op, P, M, N, K, layout):
    compare(op, P, M, N, K, layout, api.DTYPE_E4M3)
