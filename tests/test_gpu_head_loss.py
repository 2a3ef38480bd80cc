"""Cross entropy of the output layer, forward and backward, against its definition in 64 bits.

Tolerances.  Products of BF16 values are exact in FP32; the tensor cores add 16 of them to an FP32 sum at a time, each
addition off by at most 2^-23 of the sizes involved: a contraction of length k is off by (k / 8 + 4) * 2^-23 * sum |terms|
(logits: Z below).  exp and log add 2^-21 relative, the FP32 epilogue a few units of 2^-23 of the numbers it adds.  The
logits' gradient is rounded to BF16 once (8 significand bits: 2^-8 relative) before its two products, and a result in BF16
once more.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
KIND = {"bf16": api.DTYPE_BF16, "fp32": api.DTYPE_FP32}
T = {"bf16": torch.bfloat16, "fp32": torch.float32}


def split_rows(t, P):
    m = t.shape[0] // P
    return [t[r * m:(r + 1) * m].clone() for r in range(P)]


def split_vocab(t, P):
    out, v = [], 0
    for r in range(P):
        n = api.vocab_shard_rows(t.shape[0], P, r)
        out.append(t[v:v + n].clone())
        v += n
    return out


def inputs(M, hidden, vocab, ignored, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = (torch.randn(vocab, hidden, generator=g, device="cuda") * (1.5 / hidden ** 0.5)).bfloat16()
    y = torch.randint(0, vocab, (M,), generator=g, device="cuda")
    pull = torch.rand(M, 1, generator=g, device="cuda") * 5
    x = (torch.randn(M, hidden, generator=g, device="cuda") + pull * w[y].float()).bfloat16()
    off = torch.rand(M, generator=g, device="cuda") < ignored
    y[off] = torch.tensor([-1, -100, vocab, 2 ** 31 - 1], device="cuda")[torch.randint(0, 4, (M,), generator=g, device="cuda")][off]
    dloss = torch.randn(M, generator=g, device="cuda") * 1e-3
    return x, w, y, dloss


def definition(x, w, y, scale, smoothing):
    """z, Z (what |terms| of its sums add up to), lse, loss and which rows take part, in 64 bits."""
    xd, wd = x.double(), w.double()
    z = xd @ wd.T * scale
    Z = xd.abs() @ wd.abs().T * abs(scale)
    part = (y >= 0) & (y < w.shape[0])
    lse = torch.logsumexp(z, 1)
    zt = z.gather(1, y.clamp(0, w.shape[0] - 1)[:, None])[:, 0]
    loss = lse - (1 - smoothing) * zt - smoothing * z.mean(1)
    zero = torch.zeros_like(lse)
    return z, Z, torch.where(part, lse, zero), torch.where(part, loss, zero), part


def within(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {(got - want).abs()[bad].max():.3g}, its bound {bound[bad].max():.3g}"


CASES = [
    # P, M, hidden, vocab, ignored, scale, smoothing, grad
    (1, 1, 8, 1, 0.0, 1.0, 0.0, "bf16"),              # one word: p = 1, loss 0
    (1, 1, 64, 2, 0.0, 1.0, 0.0, "fp32"),
    (1, 7, 72, 255, 0.3, 1.0, 0.1, "bf16"),
    (2, 6, 8, 3, 0.0, -2.0, 0.0, "bf16"),
    (4, 4, 136, 5, 0.5, 1.0, 0.0, "fp32"),            # shards of 2, 2, 1 and 0 rows
    (16, 16, 264, 1000, 0.2, 0.5, 0.2, "bf16"),
    (1, 16, 4096, 32000, 0.0, 1.0, 0.0, "bf16"),      # few rows, more tiles than SMs
    (5, 35, 200, 2600, 0.1, 1.0, 0.1, "bf16"),        # shards of 520 rows: tiles of 8 rows, and a half without any
    (1, 64, 96, 40000, 0.0, 1.0, 0.0, "bf16"),        # two tiles and more per SM, the most of few rows
    (1, 65, 96, 40000, 0.0, 1.0, 0.0, "bf16"),        # one more
    (1, 127, 96, 40000, 0.0, 1.0, 0.0, "bf16"),
    (1, 128, 128, 256, 0.0, 1.0, 0.0, "bf16"),        # whole tiles
    (1, 256, 256, 512, 0.0, 1.0, 0.0, "fp32"),
    (3, 129, 520, 257, 0.0, 1.0, 0.0, "bf16"),        # one more than a tile
    (1, 257, 1032, 5001, 0.1, 1.0, 0.0, "bf16"),
    (8, 512, 1024, 4099, 0.0, 1.0, 0.1, "bf16"),
    (1, 513, 64, 30001, 0.9, 1.0, 0.0, "bf16"),
    (1, 600, 256, 700, 0.0, 0.0, 0.0, "bf16"),        # scale 0: a uniform distribution
    (2, 2050, 1024, 10007, 0.05, 1.0, 0.0, "fp32"),   # 512-row tiles of the logits and of dW
    (4, 4100, 2600, 12000, 0.0, 1.0, 0.0, "bf16"),    # and of dX
    (1, 8000, 320, 33333, 0.02, 1.0, 0.05, "bf16"),   # pieces of the vocabulary
]


@pytest.mark.parametrize("P,M,hidden,vocab,ignored,scale,smoothing,grad", CASES)
def test_loss_and_gradients(P, M, hidden, vocab, ignored, scale, smoothing, grad):
    x, w, y, dloss = inputs(M, hidden, vocab, ignored, M + vocab)
    h = api.make_head(P, M, hidden, vocab, logit_scale=scale, label_smoothing=smoothing, grad_dtype=KIND[grad])
    X, W = split_rows(x, P), split_vocab(w, P)
    loss, lse = (torch.full((M,), float("nan"), device="cuda") for _ in range(2))
    ws = api.alloc_head_workspace(h)
    ws[256:].random_(0, 256)                # the workspace may hold anything, NaN patterns among it
    api.compass_head_loss(h, X, W, y, loss, lse, ws)
    assert api.compass_read_status(ws) == (api.OK, 0)
    z, Z, want_lse, want_loss, part = definition(x, w, y, scale, smoothing)
    k = (hidden / 8 + 4) * U
    err_z = k * Z + 4 * U * z.abs()
    top = err_z.max(1).values
    within(lse, want_lse, torch.where(part, top + 8 * U * (z.abs().max(1).values + want_lse.abs() + 1), 0.0), "lse")
    within(loss, want_loss, torch.where(part, 3 * top + 24 * U * (z.abs().max(1).values + want_lse.abs() + 1), 0.0), "loss")

    dX = [torch.full((M // P, hidden), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(P)]
    dW = [torch.full_like(t, float("nan"), dtype=T[grad]) for t in W]
    ws = api.alloc_head_workspace(h, backward=True)
    ws[256:].random_(0, 256)
    api.compass_head_loss_backward(h, X, W, y, lse, dloss, dX, dW, ws)
    assert api.compass_read_status(ws) == (api.OK, 0)
    p = torch.exp(z - lse.double()[:, None])
    d = p - smoothing / vocab
    d[part, y[part]] -= 1 - smoothing
    g = (dloss.double() * part)[:, None]
    d *= g
    # off by the logits' error, by exp and the FP32 subtraction, by the rounding to BF16
    err_d = g.abs() * (p * (err_z + 8 * U * (z.abs() + lse.double().abs()[:, None] + 1)) + 4 * U) + 2.0 ** -8 * 1.01 * d.abs()
    half = 2.0 ** -8 * 1.01
    for got, want, size, err, n, half_unit, what in (
            (torch.cat(dX), d @ w.double() * scale, d.abs() @ w.double().abs(), err_d @ w.double().abs(), vocab, half, "dX"),
            (torch.cat(dW), d.T @ x.double() * scale, d.abs().T @ x.double().abs(), err_d.T @ x.double().abs(), M,
             half if grad == "bf16" else U, "dW")):
        # (pieces and splits of the vocabulary add at most 200 FP32 sums more)
        s = abs(scale)
        within(got, want, (half_unit + 4 * U) * want.abs() + s * err * 1.01 + s * ((n / 8 + 204) * U) * size, what)
    assert all((t[~m] == 0).all() for t, m in zip(dX, part.reshape(P, M // P)))


def run_both(h, X, W, y, dloss, ws=None):
    M = y.numel()
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    dX = [torch.empty_like(t) for t in X]
    dW = [torch.empty_like(t, dtype=T["fp32" if h.grad_dtype else "bf16"]) for t in W]
    ws = ws or (api.alloc_head_workspace(h), api.alloc_head_workspace(h, backward=True))
    api.compass_head_loss(h, X, W, y, loss, lse, ws[0])
    api.compass_head_loss_backward(h, X, W, y, lse, dloss, dX, dW, ws[1])
    return [loss, lse, *dX, *dW]


def test_rows_that_take_no_part_reach_nothing():
    """NaN and infinities in their X, lse and dloss; the others' results do not change by a bit when they are left out."""
    x, w, y, dloss = inputs(700, 256, 3000, 0.4, 5)
    off = (y < 0) | (y >= 3000)
    x[off] = float("nan")
    x[off.nonzero()[0]] = float("inf")
    dloss[off] = float("nan")
    h = api.make_head(1, 700, 256, 3000)
    loss, lse, dX, dW = run_both(h, [x], [w], y, dloss)
    assert torch.isfinite(torch.cat([t.float().flatten() for t in (loss, lse, dX, dW)])).all()
    assert (loss[off] == 0).all() and (lse[off] == 0).all() and (dX[off] == 0).all()
    n = int((~off).sum())
    alone = run_both(api.make_head(1, n, 256, 3000), [x[~off].contiguous()], [w], y[~off].contiguous(), dloss[~off].contiguous())
    for got, want in zip((loss[~off], lse[~off], dX[~off], dW), alone):
        assert torch.equal(got, want)


@pytest.mark.parametrize("grad", ["bf16", "fp32"])
def test_no_row_takes_part(grad):
    x, w, y, dloss = inputs(300, 64, 1000, 1.1, 6)
    assert ((y < 0) | (y >= 1000)).all()
    x[:] = float("nan")
    for t in run_both(api.make_head(2, 300, 64, 1000, grad_dtype=KIND[grad]), split_rows(x, 2), split_vocab(w, 2), y, dloss):
        assert (t == 0).all()


def test_no_rows_at_all():
    h = api.make_head(2, 0, 64, 100)
    none = [torch.empty(0, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    W = split_vocab(torch.randn(100, 64, device="cuda").bfloat16(), 2)
    out = run_both(h, none, W, torch.empty(0, device="cuda", dtype=torch.int64), torch.empty(0, device="cuda"))
    assert all((t == 0).all() for t in out[-2:])


def test_gradients_of_the_loss_alone():
    """dloss = 0 gives zeros; a NaN in one row's dloss stays in that row's dX and in dW."""
    x, w, y, dloss = inputs(40, 64, 500, 0.0, 8)
    h = api.make_head(1, 40, 64, 500)
    _, _, dX, dW = run_both(h, [x], [w], y, torch.zeros_like(dloss))
    assert (dX == 0).all() and (dW == 0).all()
    clean = run_both(h, [x], [w], y, dloss)[2]
    bad = dloss.clone()
    bad[17] = float("nan")
    dX = run_both(h, [x], [w], y, bad)[2]
    assert torch.isnan(dX[17]).all() and torch.isfinite(dX[:17]).all() and torch.isfinite(dX[18:]).all()
    # (dloss is then taken as it is, not over its largest value: other roundings, the same numbers)
    keep = torch.arange(40, device="cuda") != 17
    assert ((dX - clean)[keep].double().norm() <= 2.0 ** -7 * clean[keep].double().norm())


def test_large_and_infinite_logits():
    """Logits of several hundreds (exp overflows without the maximum), a column of -inf, a row with +inf."""
    w = torch.zeros(600, 64, device="cuda", dtype=torch.bfloat16)
    w[:, 0] = (torch.arange(600, device="cuda") % 7).bfloat16()
    w[300, 1] = float("-inf")
    x = torch.zeros(3, 64, device="cuda", dtype=torch.bfloat16)
    x[:, 0] = 100.0
    x[1, 0] = -100.0
    x[:, 1] = 1.0
    x[2, 2] = float("inf")                    # inf * 0 = NaN in every logit
    y = torch.tensor([6, 0, 5], device="cuda")
    loss, lse = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    h = api.make_head(1, 3, 64, 600)
    api.compass_head_loss(h, [x], [w], y, loss, lse, api.alloc_head_workspace(h))
    v = torch.arange(600) % 7
    v = v[torch.arange(600) != 300].double()
    want = torch.stack([torch.logsumexp(100 * v, 0), torch.logsumexp(-100 * v, 0)])
    assert (lse[:2].double().cpu() - want).abs().max() <= 600 * 4 * U
    assert (loss[:2].double().cpu() - (want - torch.tensor([600.0, 0.0]))).abs().max() <= 600 * 8 * U
    assert torch.isnan(loss[2]) and torch.isnan(lse[2])


def test_exact_logits_pin_the_statistics():
    """Integer inputs: the logits are exact, so lse and loss are right to the FP32 of the epilogue."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(-2, 3, (300, 64), generator=g, device="cuda").bfloat16()
    w = torch.randint(-2, 3, (2000, 64), generator=g, device="cuda").bfloat16()
    y = torch.randint(0, 2000, (300,), generator=g, device="cuda", dtype=torch.int32)
    h = api.make_head(1, 300, 64, 2000, logit_scale=0.25, index_dtype=api.INDEX_INT32)
    loss, lse = torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    api.compass_head_loss(h, [x], [w], y, loss, lse, api.alloc_head_workspace(h))
    z, _, want_lse, want_loss, _ = definition(x, w, y.long(), 0.25, 0.0)
    size = z.abs().max(1).values + want_lse.abs() + 1
    within(lse, want_lse, 6 * U * size, "lse")
    within(loss, want_loss, 12 * U * size, "loss")


def test_same_bits_every_time_and_in_graphs():
    x, w, y, dloss = inputs(1500, 512, 9000, 0.1, 9)
    h = api.make_head(4, 1500, 512, 9000)
    X, W = split_rows(x, 4), split_vocab(w, 4)
    ws = (api.alloc_head_workspace(h), api.alloc_head_workspace(h, backward=True))
    first = run_both(h, X, W, y, dloss, ws)
    for t in ws:
        t[256:].random_(0, 256)
    assert all(torch.equal(a, b) for a, b in zip(first, run_both(h, X, W, y, dloss, ws)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run_both(h, X, W, y, dloss, ws)
    y2 = y.roll(1)
    y.copy_(y2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        want = run_both(h, X, W, y, dloss)
    torch.cuda.current_stream().wait_stream(side)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(captured, want))
    assert api.compass_read_status(ws[1]) == (api.OK, 0)


def test_gradient_is_the_difference_quotient():
    """Central differences of sum(loss * g), losses from the 64-bit definition, along directions of X and W.  The quotient is
    off by its step squared times the third derivative (1e-4 of its size here), the gradients by their BF16 roundings: 2^-8
    relative for every logit's gradient and result, so by at most 2^-7 of sum |terms|."""
    x, w, y, dloss = inputs(60, 64, 300, 0.2, 10)
    h = api.make_head(1, 60, 64, 300, logit_scale=0.7, label_smoothing=0.1, grad_dtype=api.DTYPE_FP32)
    _, _, dX, dW = run_both(h, [x], [w], y, dloss)
    g = torch.Generator(device="cuda").manual_seed(2)
    for at, grad in ((0, dX), (1, dW)):
        D = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)
        values = []
        for s in (1e-3, -1e-3):
            args = [x.double(), w.double()]
            args[at] = args[at] + s * D
            values.append((definition(*args, y, 0.7, 0.1)[3] * dloss.double()).sum().item())
        slope = (values[0] - values[1]) / 2e-3
        size = (grad.double() * D).abs().sum().item()
        assert abs(slope - (grad.double() * D).sum().item()) <= 2.0 ** -7 * size


def test_offsets_beyond_32_bits():
    """A table of more than 2^32 bytes: its last rows are read and written."""
    V, H = 140_000, 16384
    w = torch.zeros(V, H, device="cuda", dtype=torch.bfloat16)
    w[V - 1, :2] = 1.0
    x = torch.zeros(2, H, device="cuda", dtype=torch.bfloat16)
    x[:, 0] = torch.tensor([3.0, 4.0], device="cuda")
    y = torch.tensor([V - 1, 0], device="cuda")
    h = api.make_head(1, 2, H, V)
    loss, lse, dX, dW = run_both(h, [x], [w], y, torch.ones(2, device="cuda"))
    n = float(V - 1)
    z = np.array([3.0, 4.0])
    want = np.log(n + np.exp(z))
    assert np.abs(lse.double().cpu().numpy() - want).max() <= 40 * U
    assert np.abs(loss.double().cpu().numpy() - (want - [3.0, 0.0])).max() <= 40 * U
    p = np.exp(z - want)
    got = dW[V - 1, 0].item()
    exact = (p[0] - 1) * 3 + p[1] * 4
    assert abs(got - exact) <= 2.0 ** -7 * abs(exact)
    assert abs(dX[0, 1].item() - (p[0] - 1)) <= 2.0 ** -7 and (dX[:, 2:] == 0).all()
    assert (dW[1:V - 1, 0].double() - (3 * np.exp(-want[0]) + 4 * np.exp(-want[1]))).abs().max() <= 2.0 ** -6 * 4e-5
