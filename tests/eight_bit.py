"""Plain forms of tensors kept in 8 bits, in 64 bits, for the tests: a power of two for each run of 128 columns of a row
(block_rows = 1) or each 128 x 128 block."""
import torch

from paper_2609_10549_b200 import api

TYPES = {api.DTYPE_E4M3: torch.float8_e4m3fn, api.DTYPE_E5M2: torch.float8_e5m2}
LARGEST = {api.DTYPE_E4M3: 448.0, api.DTYPE_E5M2: 57344.0}
BITS = {api.DTYPE_E4M3: (3, -6), api.DTYPE_E5M2: (2, -14)}      # mantissa bits, exponent of the smallest normal number


def expand(scale, rows, cols, block_rows=1):
    """Scales (bytes or float8_e8m0fnu) as one factor per element, float64."""
    b = scale.view(torch.uint8).double()
    f = torch.where(b == 255, torch.full_like(b, float("nan")), torch.exp2(b - 127))
    return f.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def values(q, scale, block_rows=1):
    """What an 8-bit matrix stands for, float64."""
    return q.double() * expand(scale, *q.shape, block_rows)


def exponents(x, format, block_rows=1):
    """The exponent of every block's scale by its definition (finite elements count)."""
    rows, cols = x.shape
    a = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).double().abs()
    br, bc = api.scale_shape(rows, cols, block_rows)
    padded = torch.zeros(br * block_rows, bc * 128, dtype=torch.float64, device=x.device)
    padded[:rows, :cols] = a
    top = padded.view(br, block_rows, bc, 128).amax((1, 3))
    e = torch.full_like(top, -127.0)
    for k in range(-127, 128):      # the smallest that fits
        e = torch.where(top > LARGEST[format] * 2.0 ** (k - 1), torch.full_like(e, float(k)), e) if k > -127 else e
    return e


def rounded(v, format):
    """Nearest number of the format (ties to even) of float64 values up to its largest; NaN stays."""
    bits, low = BITS[format]
    _, e = torch.frexp(v.abs().clamp(min=2.0 ** low))
    step = torch.exp2((e - 1 - bits).double())
    return torch.round(v / step) * step


def kept(x, format, block_rows=1):
    """(bytes of the scales, values) of a matrix kept in 8 bits, by the definition, in float64."""
    e = exponents(x, format, block_rows)
    f = torch.exp2(e).repeat_interleave(block_rows, 0)[:x.shape[0]].repeat_interleave(128, 1)[:, :x.shape[1]]
    v = x.double()
    v = torch.where(torch.isfinite(v), v, torch.full_like(v, float("nan")))
    return (e + 127).to(torch.uint8), rounded(v / f, format) * f


def random_8bit(rows, cols, format, g, block_rows=1, spread=3, whole=False):
    """A random 8-bit matrix and its scales.  `whole`: small whole numbers, so that products are exact in FP32."""
    shape = api.scale_shape(rows, cols, block_rows)
    if whole:
        q = torch.randint(-2, 3, (rows, cols), generator=g, device="cuda").float()
        spread = 1
    else:
        q = torch.randn(rows, cols, generator=g, device="cuda") * 8
    s = torch.randint(127 - spread, 128 + spread, shape, generator=g, device="cuda", dtype=torch.uint8)
    return q.to(TYPES[format]), s.view(torch.float8_e8m0fnu)


def guarded(rows, cols, dtype):
    """A tensor of NaN between two runs of guard elements, and a check that those are as they were."""
    pad = 256
    whole = torch.full((rows * cols + 2 * pad,), 77.0, device="cuda").to(dtype)
    view = whole[pad:pad + rows * cols].view(rows, cols)
    view.fill_(float("nan"))
    return view, lambda: bool((whole[:pad].float() == 77).all() and (whole[pad + rows * cols:].float() == 77).all())
