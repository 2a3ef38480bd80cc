"""Root-mean-square norm, tensors in 8 bits, their products and weight gradients: what the C ABI and the binding refuse (no GPU)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api

# Addresses that are never read: every call below is refused on the host.
A, ODD, HALF = 0x10000, 0x10001, 0x10008


def ptrs(*p):
    return (C.c_void_p * len(p))(*p)


GOOD, NULL = ptrs(A, A), ptrs(A, None)

PROBLEMS = [
    (dict(op=2), api.ERR_INVALID_ARG), (dict(P=0), api.ERR_INVALID_ARG), (dict(P=17), api.ERR_UNSUPPORTED), (dict(M=0), api.ERR_SHAPE),
    (dict(M=5), api.ERR_SHAPE), (dict(N=0), api.ERR_SHAPE), (dict(K=-16), api.ERR_SHAPE), (dict(M=2 ** 31), api.ERR_UNSUPPORTED),
    (dict(N=2 ** 31), api.ERR_UNSUPPORTED), (dict(dtype=api.DTYPE_BF16), api.ERR_UNSUPPORTED), (dict(dtype=7), api.ERR_UNSUPPORTED),
    (dict(rs_variant=api.RS_RING_RMW), api.ERR_UNSUPPORTED), (dict(b_layout=2), api.ERR_INVALID_ARG), (dict(K=24), api.ERR_ALIGNMENT),
]


def problem(**change):
    return api.make_problem(**{**dict(op=api.OP_AG_GEMM, P=2, M=4, N=16, K=32, dtype=api.DTYPE_E4M3), **change})


@pytest.mark.parametrize("change,status", PROBLEMS)
def test_problems_that_are_refused(change, status):
    assert api.compass_8bit_workspace_bytes(problem()) >= api.STATUS_BYTES
    with pytest.raises(api.CompassError) as e:
        api.compass_8bit_workspace_bytes(problem(**change))
    assert e.value.status == status
    L, g = api.lib(), problem(**change)
    for call in (L.compass_ag_gemm_8bit, L.compass_gemm_rs_8bit):
        if change.get("op") != 2:
            g.op = api.OP_GEMM_RS if call is L.compass_gemm_rs_8bit else api.OP_AG_GEMM
        assert call(C.byref(g), GOOD, GOOD, GOOD, GOOD, GOOD, A, 256, None) == status
    assert L.compass_weight_grad_8bit(C.byref(g), 0, 0, GOOD, GOOD, GOOD, GOOD, A, 256, None) == status


def test_the_other_dtypes_are_still_refused():
    """The 8-bit types are known where an entry point names them and nowhere else."""
    with pytest.raises(api.CompassError):
        api.compass_workspace_bytes(problem())
    for d in (api.DTYPE_E4M3, api.DTYPE_E5M2):
        for bad in (api.make_layer_norm(1, 1, 16, dtype=d), api.make_layer_norm(1, 1, 16, param_dtype=d)):
            with pytest.raises(api.CompassError):
                api.compass_layer_norm_workspace_bytes(bad)
            with pytest.raises(api.CompassError):
                api.compass_rms_norm_workspace_bytes(bad)


def test_products_that_are_refused():
    L = api.lib()
    for op, call in ((api.OP_AG_GEMM, L.compass_ag_gemm_8bit), (api.OP_GEMM_RS, L.compass_gemm_rs_8bit)):
        g = problem(op=op)

        def run(a=GOOD, sa=GOOD, b=GOOD, sb=GOOD, c=GOOD, ws=A, n=256, p=g):
            return call(C.byref(p), a, sa, b, sb, c, ws, n, None)

        assert call(None, GOOD, GOOD, GOOD, GOOD, GOOD, A, 256, None) == api.ERR_INVALID_ARG
        assert run(p=problem(op=1 - op)) == api.ERR_INVALID_ARG
        for name in ("a", "sa", "b", "sb", "c"):
            assert run(**{name: None}) == run(**{name: NULL}) == api.ERR_INVALID_ARG
        assert run(ws=None) == api.ERR_INVALID_ARG
        assert run(a=ptrs(A, HALF)) == run(b=ptrs(HALF, A)) == run(c=ptrs(A, ODD)) == run(ws=A + 128) == api.ERR_ALIGNMENT
        assert run(n=255) == api.ERR_BUFFER_TOO_SMALL
        assert run(p=problem(op=op, N=24, b_layout=api.B_KN)) == api.ERR_ALIGNMENT


def test_weight_gradients_that_are_refused():
    L, g = api.lib(), problem()

    def run(d=GOOD, x=GOOD, sx=GOOD, w=GOOD, ws=A, n=256, p=g, kind=api.DTYPE_BF16):
        return L.compass_weight_grad_8bit(C.byref(p), kind, 0, d, x, sx, w, ws, n, None)

    assert L.compass_weight_grad_8bit(None, 0, 0, GOOD, GOOD, GOOD, GOOD, A, 256, None) == api.ERR_INVALID_ARG
    for name in ("d", "x", "sx", "w"):
        assert run(**{name: None}) == run(**{name: NULL}) == api.ERR_INVALID_ARG
    assert run(ws=None) == api.ERR_INVALID_ARG
    assert run(d=ptrs(A, HALF)) == run(x=ptrs(HALF, A)) == run(w=ptrs(A, HALF)) == run(ws=A + 8) == api.ERR_ALIGNMENT
    assert run(n=0) == api.ERR_BUFFER_TOO_SMALL
    assert run(kind=api.DTYPE_E4M3) == run(kind=9) == api.ERR_UNSUPPORTED
    assert run(p=problem(b_layout=api.B_KN)) == api.ERR_UNSUPPORTED
    assert run(p=problem(N=12)) == api.ERR_ALIGNMENT


QUANTS = [
    (dict(P=0), api.ERR_INVALID_ARG), (dict(P=17), api.ERR_UNSUPPORTED), (dict(M=-2), api.ERR_SHAPE), (dict(M=5), api.ERR_SHAPE),
    (dict(cols=0), api.ERR_SHAPE), (dict(cols=2 ** 31), api.ERR_UNSUPPORTED), (dict(dtype=api.DTYPE_E4M3), api.ERR_UNSUPPORTED),
    (dict(format=api.DTYPE_FP32), api.ERR_UNSUPPORTED), (dict(block_rows=64), api.ERR_INVALID_ARG), (dict(cols=40), api.ERR_ALIGNMENT),
]


@pytest.mark.parametrize("change,status", QUANTS)
def test_conversions_that_are_refused(change, status):
    L, q = api.lib(), api.make_quant(**{**dict(P=2, M=4, cols=32), **change})
    for call in (L.compass_quantize, L.compass_dequantize):
        assert call(C.byref(q), GOOD, GOOD, GOOD, None) == status


def test_conversions_of_what_is_not_there():
    L, q = api.lib(), api.make_quant(2, 4, 32)
    for call in (L.compass_quantize, L.compass_dequantize):
        assert call(None, GOOD, GOOD, GOOD, None) == api.ERR_INVALID_ARG
        for i in range(3):
            for bad in (None, NULL):
                assert call(C.byref(q), *[bad if k == i else GOOD for k in range(3)], None) == api.ERR_INVALID_ARG
    x, eight = ptrs(A, HALF), ptrs(A, ODD)
    assert L.compass_quantize(C.byref(q), x, GOOD, GOOD, None) == L.compass_quantize(C.byref(q), GOOD, eight, GOOD, None) == api.ERR_ALIGNMENT
    assert L.compass_dequantize(C.byref(q), GOOD, GOOD, x, None) == L.compass_dequantize(C.byref(q), eight, GOOD, GOOD, None) == api.ERR_ALIGNMENT


def test_norms_that_are_refused():
    n, L = api.make_rms_norm(2, 4, 32), api.lib()
    need = api.compass_rms_norm_workspace_bytes(n)

    def forward(x=GOOD, r=None, g=A, s=None, y=GOOD, f=api.DTYPE_E4M3, y8=None, sc=None, rstd=None, n=n):
        return L.compass_rms_norm(C.byref(n), x, r, g, s, y, f, y8, sc, rstd, None)

    def back(dy=GOOD, x=GOOD, g=A, rstd=A, ds=None, dx=GOOD, dg=A, ws=A, size=need):
        return L.compass_rms_norm_backward(C.byref(n), dy, x, g, rstd, ds, dx, dg, ws, size, None)

    assert forward(x=None) == forward(x=NULL) == forward(y=None) == forward(y=NULL) == forward(r=GOOD) == forward(s=GOOD) == api.ERR_INVALID_ARG
    assert forward(y8=GOOD) == forward(sc=GOOD) == forward(y8=NULL, sc=GOOD) == api.ERR_INVALID_ARG
    assert forward(y8=GOOD, sc=GOOD, f=api.DTYPE_BF16) == api.ERR_UNSUPPORTED
    odd, half = ptrs(A, ODD), ptrs(A, HALF)
    assert forward(x=odd) == forward(r=odd, s=GOOD) == forward(g=ODD) == forward(rstd=A + 2) == api.ERR_ALIGNMENT
    assert forward(x=half, y8=GOOD, sc=GOOD) == forward(y8=half, sc=GOOD) == forward(g=HALF, y8=GOOD, sc=GOOD) == api.ERR_ALIGNMENT
    assert forward(n=api.make_rms_norm(2, 4, 40), y8=GOOD, sc=GOOD) == api.ERR_ALIGNMENT
    assert forward(n=api.make_rms_norm(2, 4, 32, eps=-1.0)) == forward(n=api.make_rms_norm(2, 4, 32, eps=float("nan"))) == api.ERR_INVALID_ARG
    assert back(dy=None) == back(x=NULL) == back(dx=None) == back(rstd=None) == back(ws=None) == back(ds=NULL) == api.ERR_INVALID_ARG
    assert back(ds=odd) == back(dg=ODD) == back(ws=A + 16) == api.ERR_ALIGNMENT
    assert back(size=need - 1) == api.ERR_BUFFER_TOO_SMALL


def test_struct_layout_matches_the_header():
    assert C.sizeof(api.Quant) == 4 * 4 + 2 * 8 and api.Quant.cols.offset == 24


@pytest.fixture
def here(monkeypatch):
    api.lib()
    monkeypatch.setattr(api, "_current_device", lambda: -1)       # the device of CPU tensors
    monkeypatch.setattr(api, "_raw_stream", lambda device: 0)


def test_the_binding_checks_tensors(here):
    """Types, shapes, numbers of shards and strides, before the library sees an address."""
    g = problem(M=4, N=32, K=160)
    a, sa = api.alloc_8bit(2, 2, 160, device="cpu")
    b, sb = api.alloc_8bit(2, 32, 160, block_rows=128, device="cpu")
    out = [torch.zeros(4, 32, dtype=torch.bfloat16) for _ in range(2)]
    ws = torch.zeros(256, dtype=torch.uint8)
    assert sa[0].shape == (2, 2) and sb[0].shape == (1, 2)
    wrong = [
        dict(A=a[:1]), dict(A=[t.to(torch.float8_e5m2) for t in a]), dict(A_scale=[s.view(torch.uint8) for s in sa]), dict(A_scale=[s[:1] for s in sa]),
        dict(B=[t.T for t in b]), dict(B_scale=sa), dict(Cout=[o.float() for o in out]), dict(Cout=[o[:, :16] for o in out]), dict(Cout=out[:1]),
    ]
    for change in wrong:
        with pytest.raises(ValueError):
            api.compass_ag_gemm_8bit(g, **{**dict(A=a, A_scale=sa, B=b, B_scale=sb, Cout=out, workspace=ws), **change})
    g.dtype = api.DTYPE_BF16
    with pytest.raises(ValueError, match="8-bit type"):
        api.compass_ag_gemm_8bit(g, a, sa, b, sb, out, ws)
    g.dtype = api.DTYPE_E4M3
    x, sx = api.alloc_8bit(2, 2, 160, device="cpu")
    dw = [torch.zeros(32, 160, dtype=torch.bfloat16) for _ in range(2)]
    for change in (dict(grad_dtype=api.DTYPE_FP32), dict(G=[o[:2] for o in out]), dict(dW=dw[:1]), dict(X=b)):
        with pytest.raises(ValueError):
            api.compass_weight_grad_8bit(g, **{**dict(G=out, X=x, X_scale=sx, dW=dw, workspace=ws), **change})
    n = api.make_rms_norm(2, 4, 160)
    rows = [torch.zeros(2, 160, dtype=torch.bfloat16) for _ in range(2)]
    for change in (dict(Y8=x), dict(Y8=x, scale=sb), dict(Y8=x, scale=sx, format=api.DTYPE_E5M2), dict(Y=rows[:1]), dict(rstd=torch.zeros(2))):
        with pytest.raises((ValueError, api.CompassError)):
            api.compass_rms_norm(n, **{**dict(X=rows, gamma=None), **change})
    q = api.make_quant(2, 4, 160, block_rows=0)
    with pytest.raises(ValueError):
        api.compass_quantize(q, rows, x, sx)


def test_no_ranks(here):
    ws = torch.zeros(256, dtype=torch.uint8)
    for call in (lambda: api.compass_ag_gemm_8bit(problem(P=0), [], [], [], [], [], ws), lambda: api.compass_weight_grad_8bit(problem(P=0), [], [], [], [], ws),
                 lambda: api.compass_rms_norm(api.make_rms_norm(0, 4, 16), [], None, Y=[]), lambda: api.compass_quantize(api.make_quant(0, 4, 16), [], [], [])):
        with pytest.raises(api.CompassError) as e:
            call()
        assert e.value.status == api.ERR_INVALID_ARG
