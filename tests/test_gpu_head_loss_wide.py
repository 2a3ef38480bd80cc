"""Output-layer loss with rows of millions of elements: forward and backward against their formulas.

X and the table are zero but for their first and last columns, small integers there, so the logits are exact and every sum has
few terms; what is left is the FP32 of the statistics (24 * 2^-23 of the numbers added) and the BF16 roundings of the logits'
gradient and of a result (2^-8 each).
"""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hidden", [1 << 20, (1 << 23) + 264])
def test_wide_rows(hidden):
    M, vocab, ends = 2, 3, [0, 7, hidden - 1]
    x = torch.zeros(M, hidden, device="cuda", dtype=torch.bfloat16)
    w = torch.zeros(vocab, hidden, device="cuda", dtype=torch.bfloat16)
    xe, we = torch.tensor([[1.0, 0, 2], [-1, 1, 1]], device="cuda"), torch.tensor([[1.0, 2, 0], [0, -1, 1], [1, 1, -1]], device="cuda")
    x[:, ends], w[:, ends] = xe.bfloat16(), we.bfloat16()
    y, dloss = torch.tensor([2, 0], device="cuda"), torch.tensor([1.0, 0.5], device="cuda")
    h = api.make_head(1, M, hidden, vocab)
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    dX, dW = torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
    api.compass_head_loss(h, [x], [w], y, loss, lse, api.alloc_head_workspace(h))
    api.compass_head_loss_backward(h, [x], [w], y, lse, dloss, [dX], [dW], api.alloc_head_workspace(h, backward=True))
    z = xe.double() @ we.double().T
    want = torch.logsumexp(z, 1)
    at = torch.arange(M, device="cuda")
    bound = 24 * 2.0 ** -23 * (z.abs().max() + want.abs().max() + 1)
    assert (lse.double() - want).abs().max() <= bound and (loss.double() - (want - z[at, y])).abs().max() <= 2 * bound
    d = torch.exp(z - want[:, None])
    d[at, y] -= 1
    d *= dloss.double()[:, None]
    for got, exact, size in ((dX, d @ we.double(), d.abs() @ we.double().abs()), (dW, d.T @ xe.double(), d.abs().T @ xe.double().abs())):
        assert ((got[:, ends].double() - exact).abs() <= 2.0 ** -7 * 1.01 * size + 1e-6).all()
        got[:, ends] = 0
        assert (got == 0).all()
