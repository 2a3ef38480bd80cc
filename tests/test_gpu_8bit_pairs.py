"""What the CTAs of a pair tell one another: many launches, one right behind the other, of tiles whose two halves end at different times."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.test_gpu_8bit_products import AG, RS
from tests.test_gpu_8bit_products import exact as product_of
from tests.test_gpu_8bit_products import inputs as product_inputs
from tests.test_gpu_8bit_weight_grad import exact as grad_of
from tests.test_gpu_8bit_weight_grad import inputs as grad_inputs

pytestmark = pytest.mark.gpu


def wrong(out, want):
    """1 on the GPU if any bit differs; the outputs are NaN afterwards, so that a call that writes nothing is seen."""
    bad = torch.zeros((), device="cuda", dtype=torch.int64)
    for o, w in zip(out, want):
        bad |= (o != w).any().long()
        o.fill_(float("nan"))
    return bad


# the second CTA of the last pair has no rows, or few of them; one tile each, and several a pair of CTAs
@pytest.mark.parametrize("op,P,M,N,K", [(AG, 1, 128, 2048, 256), (AG, 1, 129, 1024, 128), (AG, 1, 6500, 1000, 144), (AG, 3, 387, 4096, 528), (RS, 1, 1153, 2048, 272)])
def test_products_right_behind_one_another(op, P, M, N, K):
    a, b = product_inputs(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3, 20, whole=True)
    want = [e.to(torch.bfloat16) for e in product_of(op, P, a, b, api.B_NK)]
    pr = api.make_problem(op, P, M, N, K, dtype=api.DTYPE_E4M3)
    ws, bad = api.alloc_8bit_workspace(pr), torch.zeros((), device="cuda", dtype=torch.int64)
    outs = [[torch.full((M if op == AG else M // P, N), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(P)] for _ in range(10)]
    call = api.compass_ag_gemm_8bit if op == AG else api.compass_gemm_rs_8bit
    for _ in range(10):
        for out in outs:
            call(pr, [t[0] for t in a], [t[1] for t in a], [t[0] for t in b], [t[1] for t in b], out, ws)
        for out in outs:
            bad += wrong(out, want)
    assert bad.item() == 0 and api.compass_read_status(ws) == (api.OK, 0)


# one accumulator, both in turn, sums of 1024 rows, tiles of 512 rows, a contraction that pairs share
@pytest.mark.parametrize("grad", [api.DTYPE_BF16, api.DTYPE_FP32])
@pytest.mark.parametrize("op,P,M,N,K", [(AG, 1, 40, 72, 80), (AG, 1, 300, 6152, 2064), (RS, 2, 2300, 136, 272), (AG, 1, 200, 8192, 2560), (AG, 1, 4100, 264, 144), (AG, 1, 4100, 72, 80)])
def test_weight_gradients_right_behind_one_another(op, P, M, N, K, grad):
    d, x = grad_inputs(op, P, M, N, K, api.DTYPE_E4M3, 21, whole=True)
    kind = torch.float32 if grad == api.DTYPE_FP32 else torch.bfloat16
    want = [e.to(kind) for e in grad_of(op, P, d, x)]
    pr = api.make_problem(op, P, M, N, K, dtype=api.DTYPE_E4M3)
    ws, bad = api.alloc_8bit_workspace(pr), torch.zeros((), device="cuda", dtype=torch.int64)
    outs = [[torch.full((N, K), float("nan"), device="cuda", dtype=kind) for _ in range(P)] for _ in range(10)]
    for _ in range(10):
        for out in outs:
            api.compass_weight_grad_8bit(pr, d, [t[0] for t in x], [t[1] for t in x], out, ws, grad_dtype=grad)
        for out in outs:
            bad += wrong(out, want)
    assert bad.item() == 0 and api.compass_read_status(ws) == (api.OK, 0)


def test_no_launch_sees_what_the_one_before_left():
    """Products and weight gradients of inputs that change from launch to launch: a second CTA's scales or activations that the first
    one's products took too early would be those of the launch (or of the group) before."""
    P, M, N, K, sets = 1, 1100, 2048, 2064, 5
    pr = api.make_problem(AG, P, M, N, K, dtype=api.DTYPE_E4M3)
    ws, bad = api.alloc_8bit_workspace(pr), torch.zeros((), device="cuda", dtype=torch.int64)
    made = []
    for i in range(sets):
        a, b = product_inputs(AG, P, M, N, K, api.B_NK, api.DTYPE_E4M3, 30 + i, whole=True)
        d, x = grad_inputs(AG, P, M, N, K, api.DTYPE_E4M3, 40 + i, whole=True)
        made.append((a, b, d, x, [e.to(torch.bfloat16) for e in product_of(AG, P, a, b, api.B_NK)], [e.float() for e in grad_of(AG, P, d, x)]))
    c = [[torch.full((M, N), float("nan"), device="cuda", dtype=torch.bfloat16)] for _ in range(sets)]
    dw = [[torch.full((N, K), float("nan"), device="cuda")] for _ in range(sets)]
    split = lambda t: ([q for q, _ in t], [s for _, s in t])  # noqa: E731
    for _ in range(30):
        for i, (a, b, d, x, _, _) in enumerate(made):
            api.compass_ag_gemm_8bit(pr, *split(a), *split(b), c[i], ws)
        for i, (a, b, d, x, _, _) in enumerate(made):
            api.compass_weight_grad_8bit(pr, d, *split(x), dw[i], ws, grad_dtype=api.DTYPE_FP32)
        for i in range(sets):
            bad += wrong(c[i], made[i][4]) + wrong(dw[i], made[i][5])
    assert bad.item() == 0 and api.compass_read_status(ws) == (api.OK, 0)
