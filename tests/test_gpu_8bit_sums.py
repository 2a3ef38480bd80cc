"""Sums over many rows: how much the tensor cores' cut-off may take from a weight gradient."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.eight_bit import expand, random_8bit
from tests.test_gpu_8bit_weight_grad import AG, RS, run

pytestmark = pytest.mark.gpu


def positive(M, N, K, seed):
    """Gradients and activations above zero (the sums only grow), and the weight gradient in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, s = random_8bit(M, K, api.DTYPE_E4M3, g, spread=1)
    q = q.view(torch.uint8).bitwise_and(0x7F).view(q.dtype)
    d = torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
    e = torch.zeros(N, K, device="cuda", dtype=torch.float64)
    for rows in torch.arange(M, device="cuda").split(1 << 18):
        rows = slice(rows[0].item(), rows[-1].item() + 1)
        d[rows] = (torch.rand(rows.stop - rows.start, N, generator=g, device="cuda") + 0.5).bfloat16()
        e += d[rows].double().T @ (q[rows].double() * expand(s[rows], rows.stop - rows.start, K))
    return d, (q, s), e


@pytest.mark.parametrize("op,N,K,M", [(AG, 256, 256, 1 << 22), (RS, 72, 80, 4000000), (AG, 264, 272, 1 << 21)])
def test_bf16_gradients_over_millions_of_rows(op, N, K, M):
    """A sum over 65536 rows is made in 4096 steps.  Each cuts off less than 2^-23 of the sum so far, which grows evenly: 2^-12 of the
    whole at most.  The sums of 65536 rows are added in FP32 (64 of them: 2^-18).  Then comes BF16's half step, 2^-9 of the power of two below."""
    d, x, e = positive(M, N, K, 50)
    o = run(op, 1, M, N, K, api.DTYPE_E4M3, [d], [x], api.DTYPE_BF16)[0].double()
    step = torch.exp2(torch.frexp(e)[1].double() - 1 - 7)
    assert ((o - e).abs() <= step / 2 + (2.0 ** -12 + 2.0 ** -18) * e).all()


@pytest.mark.parametrize("M", [65536, 65600, 200000])
@pytest.mark.parametrize("N,K", [(520, 272), (2056, 1040)])
def test_bf16_gradients_about_the_longest_sum(N, K, M):
    """In whole numbers, so that only BF16's rounding is left: one sum, one and a little, several; with what is there added."""
    g = torch.Generator(device="cuda").manual_seed(M)
    q, s = random_8bit(M, K, api.DTYPE_E4M3, g, whole=True)
    d = torch.randint(-2, 3, (M, N), generator=g, device="cuda").bfloat16()
    e = sum(a.double().T @ (b.double() * expand(c, b.shape[0], K)) for a, b, c in zip(d.split(20000), q.split(20000), s.split(20000)))
    for op in (AG, RS):
        assert torch.equal(run(op, 1, M, N, K, api.DTYPE_E4M3, [d], [(q, s)], api.DTYPE_BF16)[0], e.bfloat16())
    old = torch.full((N, K), 5.0, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(run(AG, 1, M, N, K, api.DTYPE_E4M3, [d], [(q, s)], api.DTYPE_BF16, [old])[0], (e + 5).bfloat16())
