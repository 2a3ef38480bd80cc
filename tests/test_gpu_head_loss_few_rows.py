"""The statistics of few rows (up to 64), which have a kernel of their own: its epilogue pinned by exact logits, and the
precision of its sums.

Integer inputs make the logits exact integers below 2^24, whatever the order of the sum.  What is left is the FP32 of the
epilogue: scaling (1 rounding), exp2 (2^-21 relative), sums of positive terms, log2, the change of base, within 6 (lse) or 12
(loss) * 2^-23 of the largest numbers involved.  Label smoothing adds a sum of all logits: 32 in a row per thread, 4 warps, up to
8 tiles and 5 halvings, so at most 50 roundings of 2^-24 of the sum of their sizes.

The tensor cores' sums cut off what they cannot hold, a little per step, so precision goes with their length: over hidden = 4096
losses are 2e-6 to 4e-6 off (relative, root mean square) in one sum and 6e-7 in four added up in FP32.  The bound lies between.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api

pytestmark = pytest.mark.gpu

U = 2.0 ** -23


def losses(x, w, y, scale, smoothing, P=1):
    M, (vocab, hidden) = x.shape[0], w.shape
    h = api.make_head(P, M, hidden, vocab, logit_scale=scale, label_smoothing=smoothing)
    rows = [x[r * (M // P):(r + 1) * (M // P)].clone() for r in range(P)]
    table, v = [], 0
    for r in range(P):
        n = api.vocab_shard_rows(vocab, P, r)
        table.append(w[v:v + n].clone())
        v += n
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    ws = api.alloc_head_workspace(h)
    api.compass_head_loss(h, rows, table, y, loss, lse, ws)
    assert api.compass_read_status(ws) == (api.OK, 0)
    return loss.double(), lse.double()


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
@pytest.mark.parametrize("P", [1, 3])
@pytest.mark.parametrize("M", [1, 16, 33, 64])
def test_exact_logits(M, P, smoothing):
    """hidden = 1000: eight steps of 128, two in each of the four sums."""
    if M % P:
        M += P - M % P if M < 62 else -(M % P)
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randint(-2, 3, (M, 1000), generator=g, device="cuda").bfloat16()
    w = torch.randint(-2, 3, (2001, 1000), generator=g, device="cuda").bfloat16()
    y = torch.randint(0, 2001, (M,), generator=g, device="cuda")
    loss, lse = losses(x, w, y, 0.25, smoothing, P)
    z = x.double() @ w.double().T * 0.25
    want_lse = torch.logsumexp(z, 1)
    want = want_lse - (1 - smoothing) * z.gather(1, y[:, None])[:, 0] - smoothing * z.mean(1)
    size = z.abs().max(1).values + want_lse.abs() + 1
    assert ((lse - want_lse).abs() <= 6 * U * size).all()
    assert ((loss - want).abs() <= 12 * U * size + smoothing * 50 * 2.0 ** -24 * z.abs().mean(1)).all()


@pytest.mark.parametrize("M", [16, 64])
def test_precision(M):
    g = torch.Generator(device="cuda").manual_seed(M)
    H, V = 4096, 32000
    w = (torch.randn(V, H, generator=g, device="cuda") * (1.3 / math.sqrt(H))).bfloat16()
    y = torch.randint(0, V, (M,), generator=g, device="cuda")
    x = (torch.randn(M, H, generator=g, device="cuda") + w[y].float() * (torch.rand(M, 1, generator=g, device="cuda") * 9)).bfloat16()
    loss, lse = losses(x, w, y, 1.0, 0.0)
    z = x.double() @ w.double().T
    want_lse = torch.logsumexp(z, 1)
    want = want_lse - z.gather(1, y[:, None])[:, 0]
    assert (loss - want).norm() <= 1.5e-6 * want.norm()
    assert (lse - want_lse).norm() <= 1.5e-6 * want_lse.norm()
