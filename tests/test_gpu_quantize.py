"""Tensors to 8 bits and back on the GPU: the bits are those of the definition."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.eight_bit import TYPES, expand, guarded, kept

pytestmark = pytest.mark.gpu

FORMATS = [api.DTYPE_E4M3, api.DTYPE_E5M2]
KINDS = {api.DTYPE_BF16: torch.bfloat16, api.DTYPE_FP32: torch.float32}


def numbers(rows, cols, kind, seed):
    """Every size that occurs, zeros, whole runs of zeros, and numbers halfway between two of 8 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp2(torch.randint(-12, 12, (rows, cols), generator=g, device="cuda").float())
    x[torch.rand(rows, cols, generator=g, device="cuda") < 0.1] = 0
    x[::5, :128] = 0
    half = torch.randint(16, 32, (rows, cols), generator=g, device="cuda").float() / 16
    x = torch.where(torch.rand(rows, cols, generator=g, device="cuda") < 0.2, half, x)
    return x.to(KINDS[kind])


def run(x, P, kind, format, block_rows, stream=None):
    M, cols = x.shape
    q = api.make_quant(P, M, cols, dtype=kind, format=format, block_rows=block_rows)
    data, scale = api.alloc_8bit(P, M // P, cols, format, block_rows)
    for s in scale:
        s.view(torch.uint8).fill_(99)
    back = [guarded(M // P, cols, KINDS[kind]) for _ in range(P)]
    api.compass_quantize(q, list(x.split(M // P)), data, scale, stream=stream)
    api.compass_dequantize(q, data, scale, [b for b, _ in back], stream=stream)
    torch.cuda.synchronize()
    assert all(check() for _, check in back)
    return data, scale, [b for b, _ in back]


def check(x, P, kind, format, block_rows):
    each = x.shape[0] // P
    for shard, q, s, back in zip(x.split(each), *run(x, P, kind, format, block_rows)):
        b, v = kept(shard, format, block_rows)
        assert torch.equal(s.view(torch.uint8), b)
        got = q.double() * expand(s, *q.shape, block_rows)
        assert torch.equal(torch.nan_to_num(got, nan=1e99), torch.nan_to_num(v, nan=1e99))
        assert torch.equal(torch.nan_to_num(back.double(), nan=1e99), torch.nan_to_num(v.to(KINDS[kind]).double(), nan=1e99))


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("P,M,cols", [(1, 1, 16), (1, 1, 4096), (1, 3, 144), (2, 258, 400), (4, 1004, 1040), (16, 16, 128), (1, 2, 40000), (8, 1024, 8192)])
def test_bits(P, M, cols, kind, format, block_rows):
    check(numbers(M, cols, kind, M + cols), P, kind, format, block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("kind", list(KINDS))
def test_not_finite(kind, format, block_rows):
    """NaN and infinities become NaN and leave the others' scale alone; a block of nothing else has the smallest scale."""
    x = numbers(300, 272, kind, 5)
    x[0, 3], x[1, 130], x[2, 200:210] = float("nan"), float("inf"), -float("inf")
    x[150:, 128:256] = float("inf")
    x[7, 256:] = float("nan")
    check(x, 1, kind, format, block_rows)


@pytest.mark.parametrize("format", FORMATS)
def test_ends_of_the_range(format):
    """The largest and smallest numbers of FP32, maxima at, just below and just above what a scale holds."""
    top = {api.DTYPE_E4M3: 448.0, api.DTYPE_E5M2: 57344.0}[format]
    info = torch.finfo(torch.float32)
    firsts = [info.max, -info.max, info.tiny, info.smallest_normal / 2 ** 23, 1e-40, top, -top * (1 + 2 ** -23), top * (1 - 2 ** -24), 2.0, 1.75, 1.7500001, 0.0]
    x = torch.zeros(len(firsts), 128, device="cuda")
    x[:, 5] = torch.tensor(firsts, device="cuda")
    x[:, 6] = x[:, 5] / 3
    check(x, 1, api.DTYPE_FP32, format, 1)


def test_scales_that_are_not_numbers():
    """Scale 255 is NaN, 0 is 2^-127."""
    q = api.make_quant(1, 2, 128, dtype=api.DTYPE_FP32)
    data = torch.ones(2, 128, device="cuda").to(TYPES[api.DTYPE_E4M3])
    scale = torch.tensor([[255], [0]], dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    out = torch.empty(2, 128, device="cuda")
    api.compass_dequantize(q, [data], [scale], [out])
    assert out[0].isnan().all() and (out[1].double() == 2.0 ** -127).all()


def test_tensors_off_32_byte_boundaries():
    """16 bytes are enough."""
    x = torch.empty(10 * 144 + 8, device="cuda", dtype=torch.bfloat16)[8:].view(10, 144)
    assert x.data_ptr() % 32 == 16
    x.copy_(numbers(10, 144, api.DTYPE_BF16, 9))
    check(x, 1, api.DTYPE_BF16, api.DTYPE_E4M3, 1)
