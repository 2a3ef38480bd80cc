"""Root-mean-square norm, forward, of rows of 8193 to 16384 elements: more rows than blocks, so that each walks several."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.test_gpu_rms_norm import KINDS, check_forward, forward, make

pytestmark = pytest.mark.gpu

SIZES = [(1, 700, 12288), (2, 400, 16384), (1, 300, 8208)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("kind,param", [(api.DTYPE_BF16, api.DTYPE_BF16), (api.DTYPE_BF16, api.DTYPE_FP32), (api.DTYPE_FP32, api.DTYPE_FP32)])
@pytest.mark.parametrize("P,M,H", SIZES + [(1, 301, 8193), (1, 300, 15001)])
def test_forward(P, M, H, kind, param, residual):
    x, r, gamma = make(M, H, kind, param, H + 80, residual)
    check_forward(x, r, gamma, forward(x, r, gamma, P, kind, param), kind, None)


@pytest.mark.parametrize("format,both", [(api.DTYPE_E4M3, False), (api.DTYPE_E4M3, True), (api.DTYPE_E5M2, False)])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("P,M,H", SIZES)
def test_forward_in_8_bits(P, M, H, kind, residual, format, both):
    x, r, gamma = make(M, H, kind, api.DTYPE_FP32, H + 81, residual)
    check_forward(x, r, gamma, forward(x, r, gamma, P, kind, api.DTYPE_FP32, format, both), kind, format)
