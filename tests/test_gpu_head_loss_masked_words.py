"""A word masked out of the vocabulary by an infinite entry of its table row: its logit is -inf for every row that takes part,
its probability 0, and by the definition its gradient is finite.  Rows that take no part, and the zeros behind the last row
that does, must not turn it into NaN.

Tolerances as in test_gpu_head_loss.py: the logits' gradient is rounded to BF16 once (2^-8 relative) before the product, the
result once more, and the FP32 sums of n terms are off by (n / 8 + 4) * 2^-23 of the terms' sizes.
"""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
WORDS = (3, 299, 300)          # masked out
KIND = {"bf16": (api.DTYPE_BF16, torch.bfloat16), "fp32": (api.DTYPE_FP32, torch.float32)}


def inputs(M, hidden, vocab, live, sign, seed):
    """Column 1 of X is `sign` in every row that takes part, and of the table -sign * inf in the masked words' rows, 0 elsewhere."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, hidden, generator=g, device="cuda").bfloat16()
    w = (torch.randn(vocab, hidden, generator=g, device="cuda") * hidden ** -0.5).bfloat16()
    x[:, 1] = sign
    w[:, 1] = 0.0
    w[list(WORDS), 1] = -sign * float("inf")
    y = torch.randint(301, vocab, (M,), generator=g, device="cuda")
    off = torch.randperm(M, generator=g, device="cuda")[:M - live]
    y[off] = -100
    return x, w, y, torch.rand(M, generator=g, device="cuda") + 0.5


def run(x, w, y, dloss, grad):
    M, (vocab, hidden) = x.shape[0], w.shape
    h = api.make_head(1, M, hidden, vocab, grad_dtype=KIND[grad][0])
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    dX, dW = torch.empty_like(x), torch.empty(vocab, hidden, device="cuda", dtype=KIND[grad][1])
    ws, ws_back = api.alloc_head_workspace(h), api.alloc_head_workspace(h, backward=True)
    api.compass_head_loss(h, [x], [w], y, loss, lse, ws)
    api.compass_head_loss_backward(h, [x], [w], y, lse, dloss, [dX], [dW], ws_back)
    assert api.compass_read_status(ws) == api.compass_read_status(ws_back) == (api.OK, 0)
    return loss, lse, dX, dW


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("M,hidden,vocab,live,grad", [
    (1, 64, 600, 1, "bf16"),          # zeros behind the rows of a small batch
    (5, 64, 600, 3, "fp32"),
    (40, 72, 600, 29, "bf16"),
    (300, 64, 1000, 200, "fp32"),
    (300, 64, 1000, 256, "bf16"),     # rows that take part fill their tiles
    (900, 256, 2000, 513, "bf16"),    # tiles of 512 rows, and one of 256 with a single row
    (64, 64, 600, 0, "fp32"),         # no row takes part
])
def test_masked_words(M, hidden, vocab, live, grad, sign):
    x, w, y, dloss = inputs(M, hidden, vocab, live, sign, M)
    loss, lse, dX, dW = run(x, w, y, dloss, grad)
    part = y >= 0
    z = x.double()[:, 2:] @ w.double()[:, 2:].T + (x.double()[:, :1] * w.double()[:, 0])
    z[:, list(WORDS)] = float("-inf")
    assert torch.isfinite(loss).all() and torch.isfinite(lse).all()
    p = torch.exp(z - lse.double()[:, None])
    d = p.clone()
    d[part, y[part]] -= 1
    g = (dloss.double() * part)[:, None]
    d *= g
    size = x.double().abs() @ w.double().abs().nan_to_num(posinf=0.0).T      # sum of the sizes of a logit's terms
    err_d = g * (p * ((hidden / 8 + 12) * U * (size + lse.double().abs()[:, None] + 1)) + 4 * U) + 2.0 ** -8 * 1.01 * d.abs()
    err_d[:, list(WORDS)] = 0.0
    want = d.T @ x.double()
    half = 2.0 ** -8 * 1.01 if grad == "bf16" else U
    bound = (half + 4 * U) * want.abs() + 1.01 * (err_d.T @ x.double().abs()) + (M / 8 + 204) * U * (d.abs().T @ x.double().abs())
    bad = ~((dW.double() - want).abs() <= bound)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off in rows {bad.any(1).nonzero()[:8, 0].tolist()}"
    assert (dW[list(WORDS)] == 0).all()
    keep = torch.arange(hidden, device="cuda") != 1                          # (there 0 * inf stands in the sum over the words)
    assert torch.isfinite(dX[:, keep]).all() and (dX[~part] == 0).all()


@pytest.mark.parametrize("M,live", [(40, 29), (700, 400)])
def test_rows_left_out_change_no_bit(M, live):
    x, w, y, dloss = inputs(M, 128, 1500, live, 1.0, M + 1)
    got = run(x, w, y, dloss, "bf16")
    part = y >= 0
    alone = run(x[part].contiguous(), w, y[part].contiguous(), dloss[part].contiguous(), "bf16")
    keep = torch.arange(128, device="cuda") != 1
    for a, b in ((got[0][part], alone[0]), (got[1][part], alone[1]), (got[2][part][:, keep], alone[2][:, keep]), (got[3], alone[3])):
        assert torch.equal(a, b)
