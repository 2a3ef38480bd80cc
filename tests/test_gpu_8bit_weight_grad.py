"""Weight gradients from activations kept in 8 bits, on the GPU against 64 bits."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.eight_bit import guarded, random_8bit, values

pytestmark = pytest.mark.gpu

AG, RS = api.OP_AG_GEMM, api.OP_GEMM_RS
SHAPES = [
    (1, 1, 8, 16), (1, 1, 1000, 2064), (1, 17, 264, 144), (1, 130, 512, 512), (1, 501, 1000, 2064), (2, 254, 136, 400), (4, 4, 256, 256),
    (4, 516, 520, 656), (8, 1032, 128, 128), (16, 2064, 72, 272), (1, 3000, 256, 256), (3, 6000, 264, 272),
]


def inputs(op, P, M, N, K, format, seed, whole=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = [random_8bit(M // P if op == AG else M, K, format, g, whole=whole) for _ in range(P)]
    rows = M if op == AG else M // P
    if whole:
        d = [torch.randint(-2, 3, (rows, N), generator=g, device="cuda").bfloat16() for _ in range(P)]
    else:
        d = [torch.randn(rows, N, generator=g, device="cuda").bfloat16() for _ in range(P)]
    return d, x


def exact(op, P, d, x, magnitude=False):
    size = (lambda t: t.abs()) if magnitude else (lambda t: t)
    a, g = [size(values(*t)) for t in x], [size(t.double()) for t in d]
    a, g = ([torch.cat(a)] * P, g) if op == AG else (a, [torch.cat(g)] * P)
    return [q.T @ p for q, p in zip(g, a)]


def run(op, P, M, N, K, format, d, x, grad, old=None, ws=None, stream=None):
    pr = api.make_problem(op, P, M, N, K, dtype=format)
    ws = api.alloc_8bit_workspace(pr) if ws is None else ws
    out = [guarded(N, K, torch.float32 if grad == api.DTYPE_FP32 else torch.bfloat16) for _ in range(P)]
    if old is not None:
        for (o, _), v in zip(out, old):
            o.copy_(v)
    api.compass_weight_grad_8bit(pr, d, [t[0] for t in x], [t[1] for t in x], [o for o, _ in out], ws, grad_dtype=grad, accumulate=old is not None,
                                 stream=stream)
    assert api.compass_read_status(ws) == (api.OK, 0)
    assert all(check() for _, check in out)
    return [o for o, _ in out]


@pytest.mark.parametrize("grad", [api.DTYPE_BF16, api.DTYPE_FP32])
@pytest.mark.parametrize("op", [AG, RS])
@pytest.mark.parametrize("P,M,N,K", SHAPES)
def test_against_64_bits(op, P, M, N, K, grad):
    d, x = inputs(op, P, M, N, K, api.DTYPE_E4M3, 0)
    for o, e, s in zip(run(op, P, M, N, K, api.DTYPE_E4M3, d, x, grad), exact(op, P, d, x), exact(op, P, d, x, True)):
        # BF16's half step, and one unit of FP32 (2^-23, cut off) for every product that is added
        assert ((o.double() - e).abs() <= (2.0 ** -8 if grad == api.DTYPE_BF16 else 2.0 ** -24) * e.abs() + M * 2.0 ** -23 * s).all()


@pytest.mark.parametrize("grad", [api.DTYPE_BF16, api.DTYPE_FP32])
@pytest.mark.parametrize("op,P,M,N,K", [(AG, 1, 1500, 264, 272), (RS, 4, 2064, 520, 400)])
def test_accumulates(op, P, M, N, K, grad):
    """Added to what is there in FP32, and rounded once: whole numbers, so that only BF16's rounding is left."""
    d, x = inputs(op, P, M, N, K, api.DTYPE_E5M2, 1, whole=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    kind = torch.float32 if grad == api.DTYPE_FP32 else torch.bfloat16
    old = [torch.randint(-200, 200, (N, K), generator=g, device="cuda").to(kind) for _ in range(P)]
    for o, e, v in zip(run(op, P, M, N, K, api.DTYPE_E5M2, d, x, grad, old), exact(op, P, d, x), old):
        assert torch.equal(o, (e + v.double()).to(kind))


# few tiles of a long contraction, which several pairs of CTAs share; their boundaries inside a shard and at its ragged end
@pytest.mark.parametrize("grad", [api.DTYPE_BF16, api.DTYPE_FP32])
@pytest.mark.parametrize("op,P,M,N,K", [
    (AG, 1, 1999, 72, 80), (AG, 3, 4053, 520, 272), (RS, 4, 5552, 232, 480), (RS, 16, 4112, 264, 144), (AG, 1, 2100, 1280, 1040), (RS, 1, 3000, 1544, 768),
])
def test_shared_contraction(op, P, M, N, K, grad):
    """In whole numbers, so that only BF16's rounding is left, and added to what is there."""
    d, x = inputs(op, P, M, N, K, api.DTYPE_E4M3, 4, whole=True)
    kind = torch.float32 if grad == api.DTYPE_FP32 else torch.bfloat16
    old = [torch.full((N, K), 3.0, device="cuda", dtype=kind) for _ in range(P)]
    for o, e in zip(run(op, P, M, N, K, api.DTYPE_E4M3, d, x, grad, old), exact(op, P, d, x)):
        assert torch.equal(o, (e + 3).to(kind))


def test_long_sums_keep_fp32_precision():
    """A result in FP32 over 8192 rows is as close as FP32 arithmetic brings it: 2^-24 per addition of 1024 rows' sums is far below
    1e-6, and the tensor cores' cut-off over 1024 rows is half a unit (2^-24) per 16 of them at the sum's size on average: 64 * 2^-24 /
    (1024 / 16) steps of growing sums give about 1e-6 at most of the sum's magnitude."""
    M, N, K = 8192, 256, 256
    d, x = inputs(AG, 1, M, N, K, api.DTYPE_E4M3, 3)
    o, e = run(AG, 1, M, N, K, api.DTYPE_E4M3, d, x, api.DTYPE_FP32)[0], exact(AG, 1, d, x)[0]
    assert (o.double() - e).norm() / e.norm() < 1.5e-6


@pytest.mark.parametrize("format", [api.DTYPE_E4M3, api.DTYPE_E5M2])
def test_every_8_bit_number_and_scale(format):
    """One row each: dW is that row of activations times a gradient of one, in FP32, so every number of 8 bits times every scale comes
    through as BF16 holds it (E5M2's infinities, which the conversion to 8 bits never makes, count as numbers that are not)."""
    bits = torch.arange(256, device="cuda", dtype=torch.uint8).view(1, 256)
    kind = torch.float8_e4m3fn if format == api.DTYPE_E4M3 else torch.float8_e5m2
    for first in (0, 1, 100, 120, 127, 134, 200, 230, 254):
        scales = torch.tensor([[first, min(254, first + 7)]], dtype=torch.uint8, device="cuda")
        x = bits.view(kind), scales.view(torch.float8_e8m0fnu)
        d = torch.ones(1, 8, device="cuda", dtype=torch.bfloat16)
        got = run(AG, 1, 1, 8, 256, format, [d], [x], api.DTYPE_FP32)[0]
        want = values(*x).float().bfloat16().float().expand(8, 256)
        finite = torch.isfinite(x[0].float()).expand(8, 256)
        # (a subnormal operand of the tensor core may count as zero)
        small = want.abs() < torch.finfo(torch.bfloat16).tiny
        assert torch.equal(got[finite & ~small], want[finite & ~small])
        assert ((got - want)[finite & small].abs() <= torch.finfo(torch.bfloat16).tiny).all()
        assert got[x[0].float().isnan().expand(8, 256)].isnan().all()
    x = bits[:1, :128].contiguous().view(kind), torch.tensor([[255]], dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    assert run(AG, 1, 1, 8, 128, format, [d], [x], api.DTYPE_FP32)[0].isnan().all()
