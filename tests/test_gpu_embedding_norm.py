"""Embedding and layer norm, forward and backward, against plain 64-bit implementations on the host.

Tolerances.  A result computed in FP32 and rounded once differs from the exact one by half a unit of its type (relative
2^-9 for BF16, 2^-24 for FP32) plus the FP32 arithmetic: a sum of n terms in pieces of at most k terms in a row is off by
at most (k + n / k) * 2^-24 * sum |terms|.  Each check states its bound from these.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api

pytestmark = pytest.mark.gpu

T = {"bf16": torch.bfloat16, "fp32": torch.float32}
KIND = {"bf16": api.DTYPE_BF16, "fp32": api.DTYPE_FP32}
HALF_UNIT = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -23}     # a whole unit in the last place, relative: twice the rounding


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dtype)


def split_rows(t, P):
    """Separate allocations, one per rank."""
    m = t.shape[0] // P
    return [t[r * m:(r + 1) * m].clone() for r in range(P)]


def split_vocab(t, P):
    out, v = [], 0
    for r in range(P):
        n = api.vocab_shard_rows(t.shape[0], P, r)
        out.append(t[v:v + n].clone())
        v += n
    return out


def f64(ts):
    return torch.cat([t.double().cpu() for t in ts]).numpy() if isinstance(ts, (list, tuple)) else ts.double().cpu().numpy()


def close(got, want, bound):
    """Every element within `bound` (an array or a number); NaN exactly where wanted."""
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    same = got[ok] == want[ok]                   # equal infinities
    with np.errstate(invalid="ignore"):
        err = np.where(same, 0.0, np.abs(got[ok] - want[ok]))
    bound = np.broadcast_to(bound, want.shape)[ok]
    bad = ~(err <= bound)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.max(err[bad])} over {bound[bad][np.argmax(err[bad])]}"


# ---- embedding ------------------------------------------------------------------------------------------------------

LOOKUPS = [
    # P, M, hidden, vocab, dtype
    (1, 1, 1, 1, "bf16"),
    (1, 1, 8, 5, "fp32"),
    (2, 6, 7, 3, "bf16"),         # rows of 14 bytes
    (4, 8, 24, 5, "bf16"),        # shards of 2, 2, 1 and 0 rows
    (1, 33, 1001, 77, "fp32"),
    (3, 9, 4096, 100, "bf16"),
    (8, 4096, 520, 1000, "bf16"),  # four vectors per thread, ragged
    (16, 4800, 130, 1000, "fp32"),
]


@pytest.mark.parametrize("P,M,hidden,vocab,dtype", LOOKUPS)
@pytest.mark.parametrize("index", [api.INDEX_INT64, api.INDEX_INT32])
def test_embedding(P, M, hidden, vocab, dtype, index):
    rng = np.random.default_rng([P, M, hidden, vocab, index])
    table = dev(rng.standard_normal((vocab, hidden)), T[dtype])
    ids = rng.integers(0, vocab, M)
    ids[rng.random(M) < 0.2] = rng.choice([-1, -100, vocab, vocab + 7, 2 ** 31 - 1])
    W = split_vocab(table, P)
    Out = [torch.full((M // P, hidden), float("nan"), device="cuda", dtype=T[dtype]) for _ in range(P)]
    e = api.make_embedding(P, M, hidden, vocab, scale=1.7, dtype=KIND[dtype], index_dtype=index)
    api.compass_embedding(e, dev(ids, torch.int64 if index == api.INDEX_INT64 else torch.int32), W, Out)
    want = np.zeros((M, hidden))
    ok = (ids >= 0) & (ids < vocab)
    want[ok] = f64(table)[ids[ok]] * float(np.float32(1.7))
    close(f64(Out), want, np.abs(want) * HALF_UNIT[dtype])


def test_embedding_ids_beyond_32_bits_and_special_values():
    table = torch.tensor([[float("inf"), float("nan")], [-0.0, -3.0e38]], device="cuda")
    ids = torch.tensor([0, 2 ** 32, 2 ** 33 + 1, -2 ** 63, 1], device="cuda")
    out = [torch.empty(5, 2, device="cuda")]
    api.compass_embedding(api.make_embedding(1, 5, 2, 2, scale=2.0, dtype=api.DTYPE_FP32), ids, [table], out)
    close(f64(out), np.array([[np.inf, np.nan], [0, 0], [0, 0], [0, 0], [0, -np.inf]]), 0.0)


GRADS = [
    # P, M, hidden, vocab, dtype, grad, how the ids are spread
    (1, 1, 1, 1, "bf16", "bf16", "even"),
    (1, 1, 8, 3, "fp32", "fp32", "even"),
    (2, 64, 7, 3, "bf16", "fp32", "even"),           # runs that cross pieces, odd rows
    (4, 8, 24, 5, "bf16", "bf16", "even"),           # a shard without rows
    (1, 1000, 33, 50, "fp32", "bf16", "skewed"),
    (1, 3000, 1001, 32001, "fp32", "fp32", "skewed"),
    (8, 4096, 520, 1000, "bf16", "bf16", "skewed"),
    (8, 4096, 520, 1000, "bf16", "fp32", "one"),     # every token the same
    (2, 4096, 40, 600, "bf16", "fp32", "skewed"),    # one item per thread of the sort, and more
    (1, 4097, 40, 600, "bf16", "fp32", "skewed"),
    (2, 16384, 40, 600, "bf16", "fp32", "skewed"),
    (1, 16385, 40, 600, "bf16", "fp32", "skewed"),
    (1, 65536, 16, 700, "bf16", "fp32", "skewed"),   # the most a cluster sorts
    (1, 65537, 16, 700, "bf16", "fp32", "skewed"),   # one more: the tiled sort
    (2, 70000, 16, 70000, "fp32", "fp32", "even"),   # two passes, longer pieces
    (1, 70000, 8, 300, "bf16", "bf16", "none"),      # padding only
    (1, 40000, 8, 300000, "bf16", "fp32", "one"),    # three passes
    (1, 1100000, 8, 700, "bf16", "fp32", "skewed"),  # pieces of 2048 tokens, the most
    (8, 2048, 1024, 100001, "bf16", "bf16", "skewed"),   # 205 MB of rows, most of them zeros
    (3, 6, 256, 200000, "fp32", "fp32", "even"),     # one piece, nothing to join
    (1, 16000, 512, 190000, "bf16", "bf16", "even"),     # most tokens alone
]


def spread(rng, how, M, vocab):
    if how == "one":
        return np.full(M, vocab - 1)
    if how == "none":
        return np.full(M, -1)
    ids = rng.integers(0, vocab, M) if how == "even" else (np.exp(rng.random(M) * np.log(vocab + 1)) - 1).astype(np.int64).clip(0, vocab - 1)
    ids[rng.random(M) < 0.1] = rng.choice([-1, vocab])
    return ids


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("P,M,hidden,vocab,dtype,grad,how", GRADS)
def test_embedding_backward(P, M, hidden, vocab, dtype, grad, how, accumulate):
    rng = np.random.default_rng([P, M, hidden, vocab, accumulate])
    ids = spread(rng, how, M, vocab)
    dout = dev(rng.standard_normal((M, hidden)), T[dtype])
    before = dev(rng.standard_normal((vocab, hidden)), T[grad])
    dW = split_vocab(before if accumulate else torch.full_like(before, float("nan")), P)
    e = api.make_embedding(P, M, hidden, vocab, scale=0.3, dtype=KIND[dtype], grad_dtype=KIND[grad], accumulate=accumulate)
    ws = api.alloc_embedding_workspace(e)
    ws[256:].random_(0, 256)                         # the workspace may hold anything
    d_ids, shards = dev(ids, torch.int64), split_rows(dout, P)
    api.compass_embedding_backward(e, d_ids, shards, dW, ws)
    ok = (ids >= 0) & (ids < vocab)
    d = f64(dout)[ok]
    s = float(np.float32(0.3))
    want, size, count = np.zeros((vocab, hidden)), np.zeros((vocab, hidden)), np.zeros(vocab)
    np.add.at(want, ids[ok], d)
    np.add.at(size, ids[ok], np.abs(d))
    np.add.at(count, ids[ok], 1)
    want *= s
    if accumulate:
        want += f64(before)
    # pieces of 8 tokens, or of as many as make 512 pieces, but 2048 at most, summed one after the other
    run = 8 if M <= 4096 else min(2048, -(-M // 4096) * 8)
    steps = np.minimum(count, run) + count / run + 3
    close(f64(dW), want, np.abs(want) * HALF_UNIT[grad] + steps[:, None] * 2.0 ** -24 * (size * s + (np.abs(f64(before)) if accumulate else 0)))
    if not accumulate:
        again = [torch.empty_like(t) for t in dW]
        ws[256:].random_(0, 256)
        api.compass_embedding_backward(e, d_ids, shards, again, ws)
        assert all(torch.equal(a, b) for a, b in zip(dW, again))


def test_embedding_backward_keeps_padding_rows_out():
    """Infinities and NaN in the rows of padding tokens reach nothing."""
    dout = torch.ones(6, 16, device="cuda", dtype=torch.bfloat16)
    dout[1], dout[4] = float("nan"), float("inf")
    dW = [torch.empty(3, 16, device="cuda", dtype=torch.bfloat16)]
    e = api.make_embedding(1, 6, 16, 3)
    api.compass_embedding_backward(e, torch.tensor([2, -1, 0, 2, 3, 2], device="cuda"), [dout], dW, api.alloc_embedding_workspace(e))
    close(f64(dW), np.repeat([[1.0], [0.0], [3.0]], 16, 1), 0.0)


def test_embedding_without_tokens():
    dW = [torch.full((5, 9), float("nan"), device="cuda") for _ in range(2)]
    e = api.make_embedding(2, 0, 9, 10, dtype=api.DTYPE_FP32)
    none = [torch.empty(0, 9, device="cuda") for _ in range(2)]
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    api.compass_embedding(e, ids, dW, none)
    ws = api.alloc_embedding_workspace(e)
    api.compass_embedding_backward(e, ids, none, dW, ws)
    assert all((t == 0).all() for t in dW)
    kept = [torch.ones(5, 9, device="cuda") for _ in range(2)]
    api.compass_embedding_backward(api.make_embedding(2, 0, 9, 10, dtype=api.DTYPE_FP32, accumulate=True), ids, none, kept, ws)
    assert all((t == 1).all() for t in kept)


def test_embedding_gradient_is_the_difference_quotient():
    """sum(Out * G) changes by <dW, D> along a direction D of the table: the operator is linear, so the quotient is exact but
    for FP32 rounding (bound: terms * 2^-23 * sum of their sizes)."""
    rng = np.random.default_rng(7)
    M, H, V = 50, 12, 9
    ids = dev(rng.integers(-1, V, M), torch.int64)
    W, D, G = (dev(rng.standard_normal(s), torch.float32) for s in ((V, H), (V, H), (M, H)))
    e = api.make_embedding(1, M, H, V, scale=1.5, dtype=api.DTYPE_FP32)
    outs = []
    for t in (W + D, W - D):
        out = [torch.empty(M, H, device="cuda")]
        api.compass_embedding(e, ids, [t], out)
        outs.append(out[0])
    dW = [torch.empty(V, H, device="cuda")]
    api.compass_embedding_backward(e, ids, [G], dW, api.alloc_embedding_workspace(e))
    slope = ((outs[0].double() - outs[1].double()) / 2 * G.double()).sum().item()
    size = ((outs[0].double().abs() + outs[1].double().abs()) * G.double().abs()).sum().item()
    assert abs(slope - (dW[0].double() * D.double()).sum().item()) <= 60 * 2.0 ** -23 * size


# ---- layer norm -----------------------------------------------------------------------------------------------------

NORMS = [
    # P, M, hidden, dtype, param
    (1, 1, 1, "fp32", "fp32"),            # one element: the variance is zero
    (1, 1, 8, "bf16", "bf16"),
    (2, 6, 7, "bf16", "fp32"),
    (1, 5, 33, "fp32", "bf16"),
    (4, 8, 1000, "bf16", "bf16"),
    (1, 3, 1001, "bf16", "fp32"),
    (1, 400, 1001, "fp32", "fp32"),
    (8, 4096, 64, "bf16", "fp32"),        # several rows per block
    (8, 1000, 4096, "bf16", "fp32"),
    (1, 300, 2052, "fp32", "fp32"),
    (2, 302, 8192, "bf16", "bf16"),
    (1, 7, 8200, "bf16", "fp32"),         # wider than the backward pass's registers
    (1, 400, 9000, "bf16", "fp32"),
    (1, 301, 16400, "fp32", "fp32"),
    (1, 3, 17001, "bf16", "bf16"),
    (1, 2, 40000, "bf16", "fp32"),        # wider than the forward pass's
    (1, 2, 40001, "fp32", "bf16"),
]


def norm_inputs(P, M, hidden, dtype, param, seed=0):
    rng = np.random.default_rng([M, hidden, seed])
    x = dev(rng.standard_normal((M, hidden)) * rng.uniform(0.1, 3, (M, 1)) + rng.uniform(-2, 2, (M, 1)), T[dtype])
    r = dev(rng.standard_normal((M, hidden)), T[dtype])
    gamma = dev(1 + 0.3 * rng.standard_normal(hidden), T[param])
    beta = dev(rng.standard_normal(hidden), T[param])
    return x, r, gamma, beta


@pytest.mark.parametrize("mode", ["plain", "residual", "bare"])
@pytest.mark.parametrize("P,M,hidden,dtype,param", NORMS)
def test_layer_norm(P, M, hidden, dtype, param, mode):
    x, r, gamma, beta = norm_inputs(P, M, hidden, dtype, param)
    n = api.make_layer_norm(P, M, hidden, eps=1e-3, dtype=KIND[dtype], param_dtype=KIND[param])
    blank = lambda: [torch.full((M // P, hidden), float("nan"), device="cuda", dtype=T[dtype]) for _ in range(P)]  # noqa: E731
    Y, S = blank(), blank()
    mean, rstd = (torch.full((M,), float("nan"), device="cuda") for _ in range(2))
    X = split_rows(x, P)
    if mode == "bare":
        api.compass_layer_norm(n, X, None, None, Y)
        g, b, h = 1.0, 0.0, f64(x)
    else:
        more = dict(residual=split_rows(r, P), summed=S) if mode == "residual" else {}
        api.compass_layer_norm(n, X, gamma, beta, Y, mean=mean, rstd=rstd, **more)
        g, b, h = f64(gamma), f64(beta), f64(x)
        if mode == "residual":
            want = h + f64(r)
            close(f64(S), want, np.abs(want) * HALF_UNIT[dtype] + 2.0 ** -24 * (np.abs(h) + np.abs(f64(r))))
            h = f64(S)
    mu = h.mean(1, keepdims=True)
    c = h - mu
    sd = 1 / np.sqrt((c * c).mean(1, keepdims=True) + float(np.float32(1e-3)))
    # sums of n terms over at most 32 (40 in wide rows) a thread, then 10 halvings
    steps = (min(hidden, 48) + 12) * 2.0 ** -24
    err_mu = steps * np.abs(h).mean(1, keepdims=True) + 2.0 ** -23 * np.abs(mu)
    rel_sd = steps + 4 * 2.0 ** -24 + (2 * np.abs(c).mean(1, keepdims=True) * err_mu + err_mu ** 2) * sd ** 2
    want = c * sd * g + b
    bound = np.abs(want) * HALF_UNIT[dtype] + np.abs(g) * sd * (err_mu + np.abs(c) * (rel_sd + 2.0 ** -22)) + 2.0 ** -23 * np.abs(b)
    close(f64(Y), want, bound)
    if mode != "bare":
        close(f64(mean), mu[:, 0], err_mu[:, 0] + 1e-30)
        close(f64(rstd), sd[:, 0], (sd * rel_sd)[:, 0] * 2)


@pytest.mark.parametrize("dsum", [False, True])
@pytest.mark.parametrize("P,M,hidden,dtype,param", NORMS)
def test_layer_norm_backward(P, M, hidden, dtype, param, dsum):
    x, r, gamma, _ = norm_inputs(P, M, hidden, dtype, param, 1)
    rng = np.random.default_rng([M, hidden, 2])
    dy = dev(rng.standard_normal((M, hidden)), T[dtype])
    n = api.make_layer_norm(P, M, hidden, eps=1e-3, dtype=KIND[dtype], param_dtype=KIND[param])
    h = f64(x)
    mean = dev(h.mean(1), torch.float32)
    rstd = dev(1 / np.sqrt(h.var(1) + 1e-3), torch.float32)
    X, dY, R = split_rows(x, P), split_rows(dy, P), split_rows(r, P)
    dX = [torch.full((M // P, hidden), float("nan"), device="cuda", dtype=T[dtype]) for _ in range(P)]
    dg, db = (torch.full((hidden,), float("nan"), device="cuda", dtype=T[param]) for _ in range(2))
    ws = api.alloc_layer_norm_workspace(n)
    ws[256:].random_(0, 256)
    api.compass_layer_norm_backward(n, dY, X, gamma, mean, rstd, dX, dg, db, ws, dsum=R if dsum else None)
    mu, sd = f64(mean)[:, None], f64(rstd)[:, None]
    d, g = f64(dy), f64(gamma)
    xh = (h - mu) * sd
    # xhat is off by the rounding of h - mu and of the product
    err_xh = 2.0 ** -23 * (np.abs(h) + np.abs(mu)) * sd + 2.0 ** -23 * np.abs(xh)
    gd = d * g
    c1, c2 = gd.mean(1, keepdims=True), (gd * xh).mean(1, keepdims=True)
    steps = (min(hidden, 48) + 12) * 2.0 ** -24
    e1 = steps * np.abs(gd).mean(1, keepdims=True)
    e2 = steps * np.abs(gd * xh).mean(1, keepdims=True) + (np.abs(gd) * err_xh).mean(1, keepdims=True)
    want = sd * (gd - c1 - xh * c2) + (f64(r) if dsum else 0)
    size = sd * (np.abs(gd) + np.abs(c1) + np.abs(xh * c2)) + (np.abs(f64(r)) if dsum else 0)
    close(f64(dX), want, np.abs(want) * HALF_UNIT[dtype] + sd * (e1 + np.abs(xh) * e2 + err_xh * np.abs(c2)) + 4 * 2.0 ** -23 * size)
    # column sums: at most M / 64 rows in a row per thread, then the pieces
    col = (M / 64 + 64 + 32) * 2.0 ** -24
    close(f64(dg), (d * xh).sum(0), np.abs((d * xh).sum(0)) * HALF_UNIT[param] + (np.abs(d) * (np.abs(xh) * col + err_xh)).sum(0))
    close(f64(db), d.sum(0), np.abs(d.sum(0)) * HALF_UNIT[param] + col * np.abs(d).sum(0))
    again = [torch.empty_like(t) for t in dX]
    dg2, db2 = torch.empty_like(dg), torch.empty_like(db)
    ws[256:].random_(0, 256)
    api.compass_layer_norm_backward(n, dY, X, gamma, mean, rstd, again, dg2, db2, ws, dsum=R if dsum else None)
    assert all(torch.equal(a, b) for a, b in zip(dX + [dg, db], again + [dg2, db2]))


def test_layer_norm_in_place():
    x, r, gamma, beta = norm_inputs(1, 64, 512, "bf16", "fp32")
    n = api.make_layer_norm(1, 64, 512, param_dtype=api.DTYPE_FP32)
    Y, Y2, S, x2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), x.clone()
    mean, rstd = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    api.compass_layer_norm(n, [x], gamma, beta, [Y], residual=[r], summed=[S], mean=mean, rstd=rstd)
    api.compass_layer_norm(n, [x2], gamma, beta, [Y2], residual=[r], summed=[x2])
    assert torch.equal(Y, Y2) and torch.equal(S, x2)
    dX, dg, db, ws = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta), api.alloc_layer_norm_workspace(n)
    api.compass_layer_norm_backward(n, [Y], [S], gamma, mean, rstd, [dX], dg, db, ws, dsum=[r])
    r2 = r.clone()
    api.compass_layer_norm_backward(n, [Y], [S], gamma, mean, rstd, [r2], None, None, ws, dsum=[r2])
    assert torch.equal(dX, r2)


def test_layer_norm_rows_do_not_touch_one_another():
    """A row of NaN, one with an infinity, one of equal values (zero variance, eps = 0 as well)."""
    x = torch.randn(6, 40, device="cuda")
    x[1], x[3, 5], x[4] = float("nan"), float("inf"), 2.5
    Y = torch.empty_like(x)
    api.compass_layer_norm(api.make_layer_norm(1, 6, 40, dtype=api.DTYPE_FP32), [x], None, None, [Y])
    assert torch.isnan(Y[1]).all() and torch.isnan(Y[3]).all() and (Y[4] == 0).all() and torch.isfinite(Y[[0, 2, 5]]).all()
    alone = torch.empty_like(x[[0, 2, 5]])
    api.compass_layer_norm(api.make_layer_norm(1, 3, 40, dtype=api.DTYPE_FP32), [x[[0, 2, 5]]], None, None, [alone])
    assert torch.equal(alone, Y[[0, 2, 5]])
    api.compass_layer_norm(api.make_layer_norm(1, 6, 40, eps=0.0, dtype=api.DTYPE_FP32), [x], None, None, [Y])
    assert torch.isnan(Y[4]).all()                      # 0 * (1 / 0)


def test_layer_norm_large_offset():
    """The variance comes from centred values: an offset of 1000 standard deviations leaves it intact."""
    rng = np.random.default_rng(3)
    x = dev(1000 + rng.standard_normal((4, 4096)), torch.float32)
    rstd, mean, Y = torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(x)
    api.compass_layer_norm(api.make_layer_norm(1, 4, 4096, dtype=api.DTYPE_FP32), [x], None, None, [Y], mean=mean, rstd=rstd)
    h = f64(x)
    # an error of the mean of 60 * 2^-24 * 1000 changes the variance by its square alone
    close(f64(rstd), 1 / np.sqrt(h.var(1) + 1e-5), 2e-5)


def test_layer_norm_without_rows():
    n = api.make_layer_norm(4, 0, 100, param_dtype=api.DTYPE_FP32)
    none, f = [torch.empty(0, 100, device="cuda", dtype=torch.bfloat16) for _ in range(4)], torch.empty(0, device="cuda")
    g = torch.full((100,), float("nan"), device="cuda")
    b = g.clone()
    api.compass_layer_norm(n, none, None, None, none, mean=f, rstd=f)
    api.compass_layer_norm_backward(n, none, none, None, f, f, none, g, b, api.alloc_layer_norm_workspace(n))
    assert (g == 0).all() and (b == 0).all()


def test_layer_norm_gradient_is_the_difference_quotient():
    """Central differences of sum(Y * G) along random directions of x, gamma and beta, Y from the 64-bit definition: the
    quotient's own error is of the order step^2 = 1e-6, the FP32 gradient's of 1e-6."""
    rng = np.random.default_rng(11)
    M, H = 20, 48
    x, G, D = (rng.standard_normal((M, H)) for _ in range(3))
    gamma, beta, dgam, dbet = 1 + 0.2 * rng.standard_normal(H), rng.standard_normal(H), rng.standard_normal(H), rng.standard_normal(H)
    n = api.make_layer_norm(1, M, H, dtype=api.DTYPE_FP32)
    X, g, mean, rstd = dev(x, torch.float32), dev(gamma, torch.float32), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    Y = torch.empty_like(X)
    api.compass_layer_norm(n, [X], g, dev(beta, torch.float32), [Y], mean=mean, rstd=rstd)
    dX, dg, db = torch.empty_like(X), torch.empty_like(g), torch.empty_like(g)
    api.compass_layer_norm_backward(n, [dev(G, torch.float32)], [X], g, mean, rstd, [dX], dg, db, api.alloc_layer_norm_workspace(n))

    def value(x, gamma, beta):
        return (((x - x.mean(1, keepdims=True)) / np.sqrt(x.var(1, keepdims=True) + 1e-5) * gamma + beta) * G).sum()

    s = 1e-3
    for got, (a, b) in (((f64(dX) * D).sum(), ((x + s * D, gamma, beta), (x - s * D, gamma, beta))),
                        ((f64(dg) * dgam).sum(), ((x, gamma + s * dgam, beta), (x, gamma - s * dgam, beta))),
                        ((f64(db) * dbet).sum(), ((x, gamma, beta + s * dbet), (x, gamma, beta - s * dbet)))):
        want = (value(*a) - value(*b)) / (2 * s)
        assert abs(got - want) <= 1e-4 * np.sqrt(M * H)


# ---- streams, graphs, large offsets ---------------------------------------------------------------------------------


def test_calls_follow_their_stream_and_replay_in_graphs():
    M, H, V = 512, 256, 1000
    e = api.make_embedding(2, M, H, V, dtype=api.DTYPE_FP32)
    n = api.make_layer_norm(2, M, H, dtype=api.DTYPE_FP32)
    W = split_vocab(torch.randn(V, H, device="cuda"), 2)
    ids = torch.randint(0, V, (M,), device="cuda")
    out, Y, dX = ([torch.empty(M // 2, H, device="cuda") for _ in range(2)] for _ in range(3))
    dW = [torch.empty_like(w) for w in W]
    mean, rstd, dg, db = (torch.empty(k, device="cuda") for k in (M, M, H, H))
    we, wn = api.alloc_embedding_workspace(e), api.alloc_layer_norm_workspace(n)

    def step():
        api.compass_embedding(e, ids, W, out)
        api.compass_layer_norm(n, out, None, None, Y, mean=mean, rstd=rstd)
        api.compass_layer_norm_backward(n, Y, out, None, mean, rstd, dX, dg, db, wn)
        api.compass_embedding_backward(e, ids, dX, dW, we)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        ids.copy_(torch.randint(0, V, (M,), generator=torch.Generator().manual_seed(seed)))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000)
            step()
        torch.cuda.current_stream().wait_stream(side)
        want = [t.clone() for t in dW + [dg]]
        for t in dW + out + Y + dX + [dg]:
            t.fill_(float("nan"))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(dW + [dg], want))


def test_offsets_beyond_32_bits():
    """Tables and activations of more than 2^32 bytes and more than 2^31 elements."""
    V, H = 300_000, 8192
    table = torch.zeros(V, H, device="cuda", dtype=torch.bfloat16)
    table[V - 1], table[V - 2] = 3.0, 5.0
    ids = torch.tensor([V - 1, 0, V - 2, V - 1], device="cuda")
    out = [torch.empty(4, H, device="cuda", dtype=torch.bfloat16)]
    e = api.make_embedding(1, 4, H, V)
    api.compass_embedding(e, ids, [table], out)
    assert (out[0][:, 0].cpu() == torch.tensor([3.0, 0, 5, 3])).all() and (out[0] == out[0][:, :1]).all()
    table.fill_(1.0)
    api.compass_embedding_backward(e, ids, out, [table], api.alloc_embedding_workspace(e))
    rows = table[:, 0].cpu()
    assert rows[V - 1] == 6 and rows[V - 2] == 5 and rows[:V - 2].abs().sum() == 0 and (table[V - 1] == 6).all()
    M = V
    x = table.normal_()
    n = api.make_layer_norm(1, M, H)
    y = torch.empty_like(x)
    mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    api.compass_layer_norm(n, [x], None, None, [y], mean=mean, rstd=rstd)
    at = torch.tensor([0, 262143, 262144, M - 1], device="cuda")
    want = torch.nn.functional.layer_norm(x[at].double(), (H,))
    assert (y[at].double() - want).abs().max() <= 2.0 ** -7 * 4
    dx = torch.empty_like(x)
    api.compass_layer_norm_backward(n, [y], [x], None, mean, rstd, [dx], None, None, api.alloc_layer_norm_workspace(n), dsum=[x])
    xd = x[at].double().requires_grad_()
    torch.nn.functional.layer_norm(xd, (H,)).backward(y[at].double())
    want = xd.grad + x[at].double()
    assert (dx[at].double() - want).abs().max() <= 2.0 ** -7 * want.abs().max()


# ---- off the 16-byte boundaries -------------------------------------------------------------------------------------


def shifted(t, by=1):
    """The same values one element behind a 16-byte boundary."""
    room = torch.zeros(t.numel() + by, device=t.device, dtype=t.dtype)
    room[by:] = t.reshape(-1)
    return room[by:].view(t.shape)


@pytest.fixture
def off_boundaries(monkeypatch):
    import sys
    here = sys.modules[__name__]
    rows, vocab = split_rows, split_vocab
    monkeypatch.setattr(here, "split_rows", lambda t, P: [shifted(s) for s in rows(t, P)])
    monkeypatch.setattr(here, "split_vocab", lambda t, P: [shifted(s) for s in vocab(t, P)])


@pytest.mark.parametrize("P,M,hidden,vocab,dtype", [(2, 6, 4096, 33, "bf16"), (1, 40, 64, 33, "fp32"), (3, 9, 7, 10, "bf16")])
def test_embedding_off_boundaries(off_boundaries, P, M, hidden, vocab, dtype):
    test_embedding(P, M, hidden, vocab, dtype, api.INDEX_INT64)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("P,M,hidden,vocab,dtype,grad", [(2, 600, 64, 33, "bf16", "bf16"), (1, 300, 64, 133, "bf16", "fp32"),
                                                         (4, 400, 1001, 530, "fp32", "bf16"), (1, 5, 3, 1, "bf16", "bf16")])
def test_embedding_backward_off_boundaries(off_boundaries, P, M, hidden, vocab, dtype, grad, accumulate):
    test_embedding_backward(P, M, hidden, vocab, dtype, grad, "skewed", accumulate)


@pytest.mark.parametrize("P,M,hidden,dtype,param", [(2, 302, 4096, "bf16", "fp32"), (1, 500, 64, "fp32", "bf16"), (1, 3, 8192, "bf16", "bf16"),
                                                    (2, 4, 16384, "bf16", "fp32"), (1, 2, 40000, "fp32", "fp32")])
def test_layer_norm_off_boundaries(off_boundaries, P, M, hidden, dtype, param):
    for mode in ("plain", "residual", "bare"):
        test_layer_norm(P, M, hidden, dtype, param, mode)
    for dsum in (False, True):
        test_layer_norm_backward(P, M, hidden, dtype, param, dsum)


def test_any_pointer_off_its_boundary():
    """One tensor off a 16-byte boundary at a time: results as with all of them there, to a rounding of the last place."""
    M, H = 300, 512
    x, r, gamma, beta = norm_inputs(1, M, H, "bf16", "fp32")
    n = api.make_layer_norm(1, M, H, param_dtype=api.DTYPE_FP32)
    ws = api.alloc_layer_norm_workspace(n)
    mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")

    def run(off):
        t = {k: v.clone() for k, v in dict(x=x, r=r, g=gamma, b=beta, y=x, s=x, dx=x, dg=gamma, db=gamma).items()}
        if off:
            t[off] = shifted(t[off])
        api.compass_layer_norm(n, [t["x"]], t["g"], t["b"], [t["y"]], mean=mean, rstd=rstd, residual=[t["r"]], summed=[t["s"]])
        api.compass_layer_norm_backward(n, [t["r"]], [t["s"]], t["g"], mean, rstd, [t["dx"]], t["dg"], t["db"], ws, dsum=[t["x"]])
        return [t[k] for k in ("y", "s", "dx", "dg", "db")]

    want = run("")
    for off in ("x", "r", "g", "b", "y", "s", "dx", "dg", "db"):
        for got, w in zip(run(off), want):
            # (sums over a row in another order: FP32 roundings, which now and then turn a BF16 one)
            assert (got.double() - w.double()).norm() <= 2.0 ** -10 * w.double().norm(), off
