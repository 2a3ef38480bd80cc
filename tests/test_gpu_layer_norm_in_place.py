"""Layer norm in place, in every form the header allows: the same bits as with outputs of their own.  Rows enough that every
block walks several of them, copied ahead (whole vectors, FP32) or loaded when they are taken (odd rows of BF16)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api

pytestmark = pytest.mark.gpu

KIND = {"bf16": (api.DTYPE_BF16, torch.bfloat16), "fp32": (api.DTYPE_FP32, torch.float32)}
SIZES = [(5000, 7), (3000, 1001), (1500, 4096), (800, 8192)]      # beyond 148 blocks of as many rows as they work on side by side


def inputs(M, hidden, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return [make(M, hidden).to(KIND[dtype][1]) for _ in range(3)] + [1 + 0.2 * make(hidden), make(hidden)]


@pytest.mark.parametrize("over", ["X", "residual"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,hidden", SIZES + [(300, 8200), (300, 9001), (200, 20000), (200, 20001)])
def test_forward(M, hidden, dtype, over):
    x, r, _, gamma, beta = inputs(M, hidden, dtype, hidden)
    n = api.make_layer_norm(2, M, hidden, dtype=KIND[dtype][0], param_dtype=api.DTYPE_FP32)
    halves = lambda t: list(t.view(2, M // 2, hidden).unbind())  # noqa: E731
    S, Y, Y2 = (torch.empty_like(x) for _ in range(3))
    stats = [torch.empty(M, device="cuda") for _ in range(4)]
    api.compass_layer_norm(n, halves(x), gamma, beta, halves(Y), mean=stats[0], rstd=stats[1], residual=halves(r), summed=halves(S))
    taken = x if over == "X" else r
    api.compass_layer_norm(n, halves(x), gamma, beta, halves(Y2), mean=stats[2], rstd=stats[3], residual=halves(r), summed=halves(taken))
    assert torch.equal(taken, S) and torch.equal(Y, Y2)
    assert torch.equal(stats[0], stats[2]) and torch.equal(stats[1], stats[3])


@pytest.mark.parametrize("over", ["dY", "dsum"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,hidden", SIZES)
def test_backward(M, hidden, dtype, over):
    x, dy, dsum, gamma, _ = inputs(M, hidden, dtype, hidden + 1)
    n = api.make_layer_norm(2, M, hidden, dtype=KIND[dtype][0], param_dtype=api.DTYPE_FP32)
    halves = lambda t: list(t.view(2, M // 2, hidden).unbind())  # noqa: E731
    mean, rstd = x.float().mean(1), 1 / x.float().std(1)
    ws = api.alloc_layer_norm_workspace(n)
    dX = torch.empty_like(x)
    sums = [torch.empty(hidden, device="cuda") for _ in range(4)]
    api.compass_layer_norm_backward(n, halves(dy), halves(x), gamma, mean, rstd, halves(dX), sums[0], sums[1], ws, dsum=halves(dsum))
    taken = dy if over == "dY" else dsum
    api.compass_layer_norm_backward(n, halves(dy), halves(x), gamma, mean, rstd, halves(taken), sums[2], sums[3], ws, dsum=halves(dsum))
    assert torch.equal(taken, dX) and torch.equal(sums[0], sums[2]) and torch.equal(sums[1], sums[3])
    if over == "dY":      # and without a residual's gradient
        d = dX.clone()
        plain = torch.empty_like(x)
        api.compass_layer_norm_backward(n, halves(d), halves(x), gamma, mean, rstd, halves(plain), None, None, ws)
        api.compass_layer_norm_backward(n, halves(d), halves(x), gamma, mean, rstd, halves(d), None, None, ws)
        assert torch.equal(d, plain)
