"""Root-mean-square norm on the GPU, forward (also in 8 bits) and backward, against 64 bits."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.eight_bit import expand, guarded, kept

pytestmark = pytest.mark.gpu

KINDS = {api.DTYPE_BF16: torch.bfloat16, api.DTYPE_FP32: torch.float32}
HALF = {api.DTYPE_BF16: 2.0 ** -8, api.DTYPE_FP32: 2.0 ** -24}
EPS = 1e-5


def make(M, H, kind, param, seed, residual):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = (normal(M, H) * torch.exp(normal(M, 1))).to(KINDS[kind])
    return x, normal(M, H).to(KINDS[kind]) if residual else None, (1 + 0.1 * normal(H)).to(KINDS[param])


def forward(x, r, gamma, P, kind, param, format=None, both=False, eps=EPS):
    M, H = x.shape
    n = api.make_rms_norm(P, M, H, eps=eps, dtype=kind, param_dtype=param)
    split = lambda t: list(t.split(M // P))  # noqa: E731
    got = {}
    more = {}
    if r is not None:
        got["summed"], check_sum = guarded(M, H, KINDS[kind])
        more.update(residual=split(r), summed=split(got["summed"]))
    if format is None or both:
        got["y"], check_y = guarded(M, H, KINDS[kind])
        more.update(Y=split(got["y"]))
    if format is not None:
        q, s = api.alloc_8bit(1, M, H, format)
        s[0].view(torch.uint8).fill_(99)
        got["q"], got["s"] = q[0], s[0]
        more.update(Y8=split(q[0]), scale=split(s[0]), format=format)
    got["rstd"] = torch.full((M,), float("nan"), device="cuda")
    api.compass_rms_norm(n, split(x), gamma, rstd=got["rstd"], **more)
    torch.cuda.synchronize()
    assert r is None or check_sum()
    assert "y" not in got or check_y()
    return got


def definition(x, r, gamma, eps=EPS):
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    rstd = (h.double().square().mean(1) + eps).rsqrt()
    y = h.double() * rstd[:, None] * (1.0 if gamma is None else gamma.double())
    return h, rstd, y


def off(H):
    """Relative error of rstd: FP32 additions of positive numbers (H / 32 in a thread's or lane's chain at most, then 15 levels of a
    tree), the mean, square root and division: half a unit (2^-24) each, halved by the root."""
    return (min(H, 64) + 15 + 6) * 2.0 ** -24


def check_forward(x, r, gamma, got, kind, format):
    h, rstd, y = definition(x, r, gamma)
    H = x.shape[1]
    if r is not None:
        assert torch.equal(got["summed"], h)
    assert ((got["rstd"].double() - rstd).abs() <= off(H) * rstd).all()
    near = (off(H) + 2 * 2.0 ** -24) * y.abs()
    if "y" in got:
        assert ((got["y"].double() - y).abs() <= near + HALF[kind] * (y.abs() + near)).all()
    if format is not None:
        # the scale is that of the run's maximum, which may lie `near` to a border; values within half a step of that scale, which is at
        # most 2^-4 (2^-3) of the value, or of the smallest number of 8 bits
        v = got["q"].double() * expand(got["s"], *x.shape)
        low, high = (kept(y * f, format)[0].int() for f in (1 - off(H) - 2 ** -22, 1 + off(H) + 2 ** -22))
        b = got["s"].view(torch.uint8).int()
        assert ((low <= b) & (b <= high)).all()
        step, least = (2.0 ** -4, 2.0 ** -10) if format == api.DTYPE_E4M3 else (2.0 ** -3, 2.0 ** -17)
        assert ((v - y).abs() <= near + torch.maximum(step * (y.abs() + near), least * expand(got["s"], *x.shape))).all()
        # and almost everywhere they are the very ones
        assert (v == kept(y, format)[1]).double().mean() > 0.999


SIZES = [(1, 1, 16), (1, 1, 4096), (2, 6, 144), (1, 5, 1001), (4, 64, 1024), (1, 150, 272), (8, 1000, 512), (1, 301, 2064), (2, 300, 8192), (1, 3, 12288), (1, 5, 16400), (1, 2, 40000)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("kind,param", [(api.DTYPE_BF16, api.DTYPE_BF16), (api.DTYPE_BF16, api.DTYPE_FP32), (api.DTYPE_FP32, api.DTYPE_FP32)])
@pytest.mark.parametrize("P,M,H", SIZES)
def test_forward(P, M, H, kind, param, residual):
    x, r, gamma = make(M, H, kind, param, H, residual)
    check_forward(x, r, gamma, forward(x, r, gamma, P, kind, param), kind, None)


@pytest.mark.parametrize("format,both", [(api.DTYPE_E4M3, False), (api.DTYPE_E4M3, True), (api.DTYPE_E5M2, False)])
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("P,M,H", [s for s in SIZES if s[2] % 16 == 0])
def test_forward_in_8_bits(P, M, H, kind, format, both):
    x, r, gamma = make(M, H, kind, api.DTYPE_FP32, H + 1, M % 2 == 0)
    check_forward(x, r, gamma, forward(x, r, gamma, P, kind, api.DTYPE_FP32, format, both), kind, format)


def test_rows_of_zeros_and_of_what_is_not_a_number():
    """Zeros stay zeros (scale 2^-127); a NaN or infinity makes its own row NaN, in 8 bits too, and no other."""
    x, _, gamma = make(6, 272, api.DTYPE_BF16, api.DTYPE_BF16, 0, False)
    x[1] = 0
    x[3, 5] = float("nan")
    got = forward(x, None, gamma, 1, api.DTYPE_BF16, api.DTYPE_BF16, api.DTYPE_E4M3, True)
    assert (got["y"][1] == 0).all() and (got["q"][1].float() == 0).all() and (got["s"][1].view(torch.uint8) == 0).all()
    assert got["y"][3].isnan().all() and got["q"][3].float().isnan().all()
    rows = [0, 2, 4, 5]
    assert torch.isfinite(got["y"][rows].float()).all() and torch.isfinite(got["q"][rows].float()).all()


def test_without_gamma_and_in_place():
    x, r, _ = make(40, 528, api.DTYPE_BF16, api.DTYPE_BF16, 1, True)
    h, rstd, y = definition(x, r, None)
    n = api.make_rms_norm(1, 40, 528, eps=EPS)
    for into in (0, 1):
        a, b = x.clone(), r.clone()
        out = torch.empty_like(x)
        api.compass_rms_norm(n, [a], None, Y=[out], residual=[b], summed=[(a, b)[into]])
        assert torch.equal((a, b)[into], h) and ((out.double() - y).abs() <= 2.0 ** -7.9 * y.abs()).all()


def backward(dy, x, gamma, rstd, ds, P, kind, param, want_gamma=True, in_place=None):
    M, H = x.shape
    n = api.make_rms_norm(P, M, H, eps=EPS, dtype=kind, param_dtype=param)
    split = lambda t: None if t is None else list(t.split(M // P))  # noqa: E731
    dx, check = guarded(M, H, KINDS[kind])
    if in_place is not None:
        dx, check = in_place, lambda: True
    dgamma = torch.full((H,), float("nan"), device="cuda", dtype=KINDS[param]) if want_gamma else None
    api.compass_rms_norm_backward(n, split(dy), split(x), gamma, rstd, split(dx), dgamma, api.alloc_rms_norm_workspace(n), dsum=split(ds))
    torch.cuda.synchronize()
    assert check()
    return dx, dgamma


def gradient(dy, x, gamma, rstd, ds):
    """dX, dgamma, and the magnitudes of what is added up in them."""
    r, up = rstd.double()[:, None], dy.double()
    xh, v = x.double() * r, up * (1.0 if gamma is None else gamma.double())
    mean, size = (v * xh).mean(1, keepdim=True), (v * xh).abs().mean(1, keepdim=True)
    dx = r * (v - xh * mean) + (0 if ds is None else ds.double())
    big = r * (v.abs() + xh.abs() * size) + (0 if ds is None else ds.double().abs())
    return dx, (up * xh).sum(0), big, (up * xh).abs().sum(0)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("kind,param", [(api.DTYPE_BF16, api.DTYPE_BF16), (api.DTYPE_BF16, api.DTYPE_FP32), (api.DTYPE_FP32, api.DTYPE_FP32)])
@pytest.mark.parametrize("P,M,H", SIZES + [(1, 2000, 1001), (1, 700, 8200), (1, 129, 8193)])
def test_backward(P, M, H, kind, param, residual):
    x, ds, gamma = make(M, H, kind, param, H + 2, residual)
    dy = torch.randn(M, H, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(KINDS[kind])
    rstd = (x.double().square().mean(1) + EPS).rsqrt().float()
    dx, dgamma = backward(dy, x, gamma, rstd, ds, P, kind, param)
    ex, eg, big, sums = gradient(dy, x, gamma, rstd, ds)
    # a row's mean: chains of at most 64 additions and a tree; five operations around it.  Columns: M additions at most.
    near = (64 + 15 + 8) * 2.0 ** -24 * big
    assert ((dx.double() - ex).abs() <= near + HALF[kind] * (ex.abs() + near)).all()
    near = (min(M, 400) + 200) * 2.0 ** -24 * sums
    assert ((dgamma.double() - eg).abs() <= near + HALF[param] * (eg.abs() + near)).all()


@pytest.mark.parametrize("H", [144, 8208])
def test_backward_in_place_and_without_gamma(H):
    x, ds, gamma = make(70, H, api.DTYPE_BF16, api.DTYPE_FP32, 3, True)
    dy = torch.randn_like(x)
    rstd = (x.double().square().mean(1) + EPS).rsqrt().float()
    want, _ = backward(dy, x, gamma, rstd, ds, 1, api.DTYPE_BF16, api.DTYPE_FP32)
    for which in (0, 1):
        a, b = dy.clone(), ds.clone()
        got, none = backward(a, x, gamma, rstd, b, 1, api.DTYPE_BF16, api.DTYPE_FP32, want_gamma=False, in_place=(a, b)[which])
        assert none is None and torch.equal(got, want)
    ones, _ = backward(dy, x, torch.ones_like(gamma), rstd, ds, 1, api.DTYPE_BF16, api.DTYPE_FP32)
    assert torch.equal(backward(dy, x, None, rstd, ds, 1, api.DTYPE_BF16, api.DTYPE_FP32)[0], ones)


def test_backward_against_differences():
    """dX and dgamma as the slopes of the norm itself (FP32, in 64 bits around the call's own forward)."""
    M, H = 4, 80
    x, _, gamma = make(M, H, api.DTYPE_FP32, api.DTYPE_FP32, 4, False)
    dy = torch.randn(M, H, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    dx, dgamma = backward(dy, x, gamma, forward(x, None, gamma, 1, api.DTYPE_FP32, api.DTYPE_FP32)["rstd"], None, 1, api.DTYPE_FP32, api.DTYPE_FP32)

    def total(a, b):
        return (definition(a, None, b)[2] * dy.double()).sum()

    g = torch.Generator(device="cuda").manual_seed(6)
    for _ in range(4):
        u, v = (torch.randn(*t.shape, generator=g, device="cuda", dtype=torch.float64) for t in (x, gamma))
        h = 1e-5
        slope = (total(x.double() + h * u, gamma.double() + h * v) - total(x.double() - h * u, gamma.double() - h * v)) / (2 * h)
        assert abs(slope - (dx.double() * u).sum() - (dgamma.double() * v).sum()) < 1e-4 * (dx.double() * u).abs().sum()


def test_no_rows():
    n = api.make_rms_norm(2, 0, 32, param_dtype=api.DTYPE_FP32)
    empty = [torch.empty(0, 32, device="cuda", dtype=torch.bfloat16)] * 2
    api.compass_rms_norm(n, empty, None, Y=empty)
    dgamma = torch.ones(32, device="cuda")
    api.compass_rms_norm_backward(n, empty, empty, None, torch.empty(0, device="cuda"), empty, dgamma, api.alloc_rms_norm_workspace(n))
    assert (dgamma == 0).all()
    q = api.make_quant(2, 0, 32)
    data, scale = api.alloc_8bit(2, 0, 32)
    api.compass_quantize(q, empty, data, scale)
    api.compass_dequantize(q, data, scale, empty)
