"""Losses and log-sum-exps of long contractions are as good as FP32 arithmetic's.

The tensor cores' sums cut off what they cannot hold at every step, so that one long sum is off in proportion to its length:
relative, root mean square, 2.5e-6 over 4096 elements and 5.5e-6 over 8192, where FP32 arithmetic in blocked sums is 4e-7 to 7e-7
off.  Sums of 1024 elements added up in FP32 are held to twice 6e-7, whatever the contraction's length.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api

pytestmark = pytest.mark.gpu

BOUND = 2 * 6e-7


@pytest.mark.parametrize("M,hidden,vocab,smoothing", [
    (16, 8192, 32000, 0.0),
    (64, 8192, 8000, 0.0),           # the most of few rows
    (65, 8192, 8000, 0.1),           # one more: pairs of CTAs
    (300, 4104, 20000, 0.0),         # five ranges, the last one of a single stage
    (2000, 4096, 32000, 0.0),
    (1024, 16384, 4000, 0.0),
    (700, 1096, 8000, 0.0),
])
def test_precision(M, hidden, vocab, smoothing):
    g = torch.Generator(device="cuda").manual_seed(hidden)
    w = (torch.randn(vocab, hidden, generator=g, device="cuda") * (1.3 / math.sqrt(hidden))).bfloat16()
    y = torch.randint(0, vocab, (M,), generator=g, device="cuda")
    x = (torch.randn(M, hidden, generator=g, device="cuda") + w[y].float() * (torch.rand(M, 1, generator=g, device="cuda") * 9)).bfloat16()
    h = api.make_head(1, M, hidden, vocab, label_smoothing=smoothing)
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    ws = api.alloc_head_workspace(h)
    ws[256:].random_(0, 256)
    api.compass_head_loss(h, [x], [w], y, loss, lse, ws)
    assert api.compass_read_status(ws) == (api.OK, 0)
    z = x.double() @ w.double().T
    want_lse = torch.logsumexp(z, 1)
    want = want_lse - (1 - smoothing) * z.gather(1, y[:, None])[:, 0] - smoothing * z.mean(1)
    for got, exact in ((lse, want_lse), (loss, want)):
        assert (got.double() - exact).norm() <= BOUND * exact.norm()


@pytest.mark.parametrize("M,hidden", [(65, 1088), (300, 4104), (1030, 9000)])
def test_exact_logits_over_several_ranges(M, hidden):
    """Integers: every range's sum and their sum are exact, so a range left out, doubled or mixed up would show."""
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randint(-2, 3, (M, hidden), generator=g, device="cuda").bfloat16()
    w = torch.randint(-2, 3, (3001, hidden), generator=g, device="cuda").bfloat16()
    y = torch.randint(0, 3001, (M,), generator=g, device="cuda")
    h = api.make_head(1, M, hidden, 3001, logit_scale=0.125)
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    api.compass_head_loss(h, [x], [w], y, loss, lse, api.alloc_head_workspace(h))
    z = x.double() @ w.double().T * 0.125
    want = torch.logsumexp(z, 1)
    size = z.abs().max(1).values + want.abs() + 1
    assert ((lse.double() - want).abs() <= 6 * 2.0 ** -23 * size).all()
    assert ((loss.double() - (want - z.gather(1, y[:, None])[:, 0])).abs() <= 12 * 2.0 ** -23 * size).all()
