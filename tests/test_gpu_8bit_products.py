"""Products of 8-bit operands with block scales on the GPU against 64 bits."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.eight_bit import guarded, random_8bit, values

pytestmark = pytest.mark.gpu

AG, RS = api.OP_AG_GEMM, api.OP_GEMM_RS


def inputs(op, P, M, N, K, layout, format, seed, **more):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = M // P if op == AG else M
    a = [random_8bit(rows, K, format, g, **more) for _ in range(P)]
    b = [random_8bit(*((K, N) if layout == api.B_KN else (N, K)), api.DTYPE_E4M3, g, block_rows=128, **more) for _ in range(P)]
    return a, b


def exact(op, P, a, b, layout, magnitude=False):
    """The product in 64 bits, and (magnitude) the same of absolute values."""
    size = (lambda x: x.abs()) if magnitude else (lambda x: x)
    x = [size(values(*t)) for t in a]
    w = [size(values(*t, block_rows=128)) for t in b]
    if layout == api.B_NK:
        w = [t.T for t in w]
    if op == AG:
        return [torch.cat(x) @ t for t in w]
    return list(sum(p @ q for p, q in zip(x, w)).chunk(P))


def run(op, P, M, N, K, layout, format, a, b, ws=None, stream=None):
    pr = api.make_problem(op, P, M, N, K, dtype=format, b_layout=layout)
    ws = api.alloc_8bit_workspace(pr) if ws is None else ws
    out = [guarded(M if op == AG else M // P, N, torch.bfloat16) for _ in range(P)]
    call = api.compass_ag_gemm_8bit if op == AG else api.compass_gemm_rs_8bit
    call(pr, [t[0] for t in a], [t[1] for t in a], [t[0] for t in b], [t[1] for t in b], [o for o, _ in out], ws, stream=stream)
    assert api.compass_read_status(ws) == (api.OK, 0)
    assert all(check() for _, check in out)
    return [o for o, _ in out]


def compare(op, P, M, N, K, layout, format, seed=0):
    a, b = inputs(op, P, M, N, K, layout, format, seed)
    out = run(op, P, M, N, K, layout, format, a, b)
    total = K * (P if op == RS else 1)
    for o, e, s in zip(out, exact(op, P, a, b, layout), exact(op, P, a, b, layout, True)):
        # BF16's half step, and one unit of FP32 (2^-23, cut off) for every product that is added
        assert ((o.double() - e).abs() <= 2.0 ** -8 * e.abs() + total * 2.0 ** -23 * s).all()
    return a, b, out


# few rows (one accumulator column each), then pairs of CTAs; every ragged edge, slices of the contraction shorter than a scale's
# block, several groups of scales, and contractions that are split over a cluster
SHAPES = [
    (1, 1, 128, 128), (1, 1, 4096, 4096), (1, 3, 200, 16), (1, 7, 129, 144), (1, 64, 512, 2064), (1, 130, 100, 528), (1, 256, 640, 1040),
    (2, 2, 96, 272), (4, 4, 1000, 640), (8, 8, 256, 256), (8, 104, 336, 400), (2, 118, 5003, 2064), (16, 16, 64, 1168),
    (1, 257, 256, 128), (1, 300, 257, 1024), (1, 513, 1000, 2064), (1, 1000, 33, 80), (2, 514, 31, 1552), (4, 1028, 4096, 656), (8, 1024, 688, 512),
    (3, 999, 1111, 1136), (16, 2064, 272, 160), (1, 2, 20000, 256), (1, 4000, 3000, 144),
]


@pytest.mark.parametrize("op", [AG, RS])
@pytest.mark.parametrize("P,M,N,K", SHAPES)
def test_against_64_bits(op, P, M, N, K):
    compare(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3)


@pytest.mark.parametrize("op", [AG, RS])
@pytest.mark.parametrize("P,M,N,K", [s for s in SHAPES if s[2] % 16 == 0])
def test_weights_along_n(op, P, M, N, K):
    compare(op, P, M, N, K, api.B_KN, api.DTYPE_E5M2)


# few tiles of a long contraction: rows in pieces, several shards a tile and a last tile of fewer, boundaries of ranks inside a tile
@pytest.mark.parametrize("layout", [api.B_NK, api.B_KN])
@pytest.mark.parametrize("op,P,M,N,K", [
    (AG, 1, 257, 80, 4112), (AG, 2, 1202, 112, 8192), (AG, 16, 640, 64, 4112), (AG, 16, 1600, 80, 6160), (AG, 5, 95, 16, 16400),
    (RS, 8, 600, 112, 2064), (RS, 3, 807, 48, 4096), (RS, 16, 4112, 16, 2048), (RS, 8, 152, 96, 3120),
])
def test_row_tiles(op, P, M, N, K, layout):
    compare(op, P, M, N, K, layout, api.DTYPE_E4M3)


@pytest.mark.parametrize("layout", [api.B_NK, api.B_KN])
@pytest.mark.parametrize("format", [api.DTYPE_E4M3, api.DTYPE_E5M2])
@pytest.mark.parametrize("op,P,M,N,K", [(AG, 2, 20, 400, 1040), (RS, 2, 20, 400, 1040), (AG, 2, 700, 400, 1040), (RS, 4, 700, 400, 528)])
def test_whole_numbers_are_exact(op, P, M, N, K, format, layout):
    """Small whole numbers and scales whose sums FP32 holds: nothing but the rounding to BF16 is left."""
    a, b = inputs(op, P, M, N, K, layout, format, 1, whole=True)
    out = run(op, P, M, N, K, layout, format, a, b)
    for o, e in zip(out, exact(op, P, a, b, layout)):
        assert torch.equal(o, e.to(torch.bfloat16))
