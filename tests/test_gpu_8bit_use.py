"""The 8-bit operators as a program may use them: numbers that are none, tensors among others, streams, graphs, two calls at once,
the same bits every time, tensors beyond 4 GB."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.eight_bit import TYPES, expand, kept, random_8bit, values
from tests.test_gpu_8bit_products import AG, RS
from tests.test_gpu_8bit_products import exact as product_of
from tests.test_gpu_8bit_products import inputs as product_inputs
from tests.test_gpu_8bit_products import run as run_product
from tests.test_gpu_8bit_weight_grad import exact as grad_of
from tests.test_gpu_8bit_weight_grad import inputs as grad_inputs
from tests.test_gpu_8bit_weight_grad import run as run_grad

pytestmark = pytest.mark.gpu

NAN = 0x7F      # in E4M3, and as a byte of scales 2^0


def among_nan(t, fill=NAN):
    """The same tensor in a buffer whose other bytes are `fill`."""
    raw = t.contiguous().view(torch.uint8).flatten()
    whole = torch.full((raw.numel() + 2 * 65536,), fill, dtype=torch.uint8, device="cuda")
    whole[65536:65536 + raw.numel()] = raw
    return whole[65536:65536 + raw.numel()].view(t.dtype).view(t.shape)


# few rows with and without a split contraction, and pairs; all with rows, columns and contractions that end inside a tile
SHAPES = [(AG, 2, 6, 200, 656), (RS, 2, 30, 1000, 144), (AG, 1, 60, 20000, 272), (AG, 2, 600, 400, 656), (RS, 3, 999, 336, 144)]


@pytest.mark.parametrize("layout", [api.B_NK, api.B_KN])
@pytest.mark.parametrize("op,P,M,N,K", SHAPES)
def test_products_read_nothing_else(op, P, M, N, K, layout):
    """Tensors among NaNs (scales among NaNs too) give the same bits."""
    N = N // 16 * 16
    a, b = product_inputs(op, P, M, N, K, layout, api.DTYPE_E4M3, 5)
    want = run_product(op, P, M, N, K, layout, api.DTYPE_E4M3, a, b)
    a2, b2 = ([(among_nan(q), among_nan(s, 255)) for q, s in t] for t in (a, b))
    for x, y in zip(want, run_product(op, P, M, N, K, layout, api.DTYPE_E4M3, a2, b2)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("grad", [api.DTYPE_BF16, api.DTYPE_FP32])
@pytest.mark.parametrize("op,P,M,N,K", [(AG, 2, 140, 264, 400), (RS, 3, 300, 72, 272), (AG, 1, 2000, 1032, 528)])
def test_weight_gradients_read_nothing_else(op, P, M, N, K, grad):
    d, x = grad_inputs(op, P, M, N, K, api.DTYPE_E4M3, 6)
    want = run_grad(op, P, M, N, K, api.DTYPE_E4M3, d, x, grad)
    d2, x2 = [among_nan(t, 255) for t in d], [(among_nan(q), among_nan(s, 255)) for q, s in x]
    for a, b in zip(want, run_grad(op, P, M, N, K, api.DTYPE_E4M3, d2, x2, grad)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("op,P,M,N,K", SHAPES)
def test_what_is_not_a_number_stays_in_its_row_or_column(op, P, M, N, K):
    a, b = product_inputs(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3, 7)
    clean = run_product(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3, a, b)
    row, col, block = 1, N - 1, 0
    a[0][0].view(torch.uint8)[row, K - 1] = NAN                  # a value of a row
    a[-1][1].view(torch.uint8)[0, 0] = 255                       # a scale
    b[0][0].view(torch.uint8)[col, 0] = NAN                      # a weight
    got = run_product(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3, a, b)
    for r in range(P):
        bad = torch.zeros_like(clean[r], dtype=torch.bool)
        if op == AG:
            rows = M // P
            bad[[row, (P - 1) * rows]] = True
            if r == 0:
                bad[:, col] = True
        else:
            first = r * (M // P)
            for i in (row, 0):
                if first <= i < first + M // P:
                    bad[i - first] = True
            bad[:, col] = True
        assert got[r][bad].isnan().all() and torch.equal(got[r][~bad], clean[r][~bad])


def test_a_gradient_that_is_not_a_number_stays_in_its_row():
    P, M, N, K = 2, 140, 264, 400
    d, x = grad_inputs(AG, P, M, N, K, api.DTYPE_E4M3, 8)
    clean = run_grad(AG, P, M, N, K, api.DTYPE_E4M3, d, x, api.DTYPE_BF16)
    d[1][3, 7] = float("inf")
    x[0][0].view(torch.uint8)[5, 300] = NAN
    got = run_grad(AG, P, M, N, K, api.DTYPE_E4M3, d, x, api.DTYPE_BF16)
    for r in range(P):
        bad = torch.zeros(N, K, dtype=torch.bool, device="cuda")
        bad[:, 300] = True
        if r == 1:
            bad[7] = True
        assert torch.equal(got[r][~bad], clean[r][~bad]) and not torch.isfinite(got[r][bad].float()).any()


def calls(seed=0):
    """One call of every operator with its inputs, outputs and what it should give."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    made = []
    for op, P, M, N, K in ((AG, 1, 1, 4096, 4096), (AG, 2, 118, 1003, 2064), (RS, 2, 700, 400, 1040), (AG, 1, 256, 512, 1024)):
        pr = api.make_problem(op, P, M, N, K, dtype=api.DTYPE_E4M3)
        a, b = product_inputs(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3, seed + M)
        out = [torch.empty(M if op == AG else M // P, N, device="cuda", dtype=torch.bfloat16) for _ in range(P)]
        ws = api.alloc_8bit_workspace(pr)
        args = [t[0] for t in a], [t[1] for t in a], [t[0] for t in b], [t[1] for t in b], out, ws
        call = api.compass_ag_gemm_8bit if op == AG else api.compass_gemm_rs_8bit
        made.append((lambda call=call, pr=pr, args=args, **k: call(pr, *args, **k), out))
    P, M, N, K = 2, 1500, 520, 656
    pr = api.make_problem(AG, P, M, N, K, dtype=api.DTYPE_E4M3)
    d, x = grad_inputs(AG, P, M, N, K, api.DTYPE_E4M3, seed)
    for kind in (api.DTYPE_BF16, api.DTYPE_FP32):
        dw = [torch.empty(N, K, device="cuda", dtype=torch.float32 if kind else torch.bfloat16) for _ in range(P)]
        ws = api.alloc_8bit_workspace(pr)
        made.append((lambda dw=dw, ws=ws, kind=kind, **k: api.compass_weight_grad_8bit(pr, d, [t[0] for t in x], [t[1] for t in x], dw, ws, grad_dtype=kind, **k), dw))
    X = [torch.randn(300, 528, generator=g, device="cuda", dtype=torch.bfloat16)]
    q = api.make_quant(1, 300, 528)
    data, scale = api.alloc_8bit(1, 300, 528)
    made.append((lambda **k: api.compass_quantize(q, X, data, scale, **k), [data[0].view(torch.uint8), scale[0].view(torch.uint8)]))
    n = api.make_rms_norm(1, 300, 528)
    y8, ys = api.alloc_8bit(1, 300, 528)
    y, rstd = [torch.empty_like(X[0])], torch.empty(300, device="cuda")
    made.append((lambda **k: api.compass_rms_norm(n, X, None, Y=y, rstd=rstd, Y8=y8, scale=ys, **k), [y[0], rstd, y8[0].view(torch.uint8), ys[0].view(torch.uint8)]))
    dx, dgamma, wn = [torch.empty_like(X[0])], torch.empty(528, device="cuda", dtype=torch.bfloat16), api.alloc_rms_norm_workspace(n)
    r2 = (X[0].double().square().mean(1) + n.eps).rsqrt().float()
    made.append((lambda **k: api.compass_rms_norm_backward(n, X, X, None, r2, dx, dgamma, wn, **k), [dx[0], dgamma]))
    return made


def outcome(made):
    torch.cuda.synchronize()
    return [[t.clone() for t in out] for _, out in made]


def same(a, b):
    return all(torch.equal(x, y) for s, t in zip(a, b) for x, y in zip(s, t))


def test_the_same_bits_every_time_and_on_any_stream():
    made = calls()
    for call, _ in made:
        call()
    want = outcome(made)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(10):
        for _, out in made:
            for t in out:
                t.zero_()
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for i, (call, _) in enumerate(made):
            call(stream=streams[(i + turn) % 2])
        assert same(outcome(made), want)


def test_two_calls_at_once():
    """Two programs' calls on two streams, each with its own tensors and workspaces, many in flight."""
    a, b = calls(1), calls(2)
    for call, _ in a + b:
        call()
    want = outcome(a), outcome(b)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for made, s in ((a, streams[0]), (b, streams[1])):
            for call, _ in made:
                call(stream=s)
    assert same(outcome(a), want[0]) and same(outcome(b), want[1])


def test_captured_and_replayed_on_new_inputs():
    made = calls(3)
    for call, _ in made:
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call, _ in made:
            call()
    want = outcome(made)
    for _, out in made:
        for t in out:
            t.zero_()
    for _ in range(3):
        graph.replay()
    assert same(outcome(made), want)


def test_one_tensor_for_several_ranks():
    """Shards, weights and scales may be the same tensors."""
    P, M, N, K = 4, 512, 256, 256
    a, b = product_inputs(AG, P, M, N, K, api.B_NK, api.DTYPE_E4M3, 9)
    a, b = [a[0]] * P, [b[0]] * P
    for o in run_product(AG, P, M, N, K, api.B_NK, api.DTYPE_E4M3, a, b):
        for chunk in o.split(M // P):
            assert torch.equal(chunk, o[:M // P])


def big(rows, cols, g):
    """A large 8-bit matrix: a random block of rows again and again."""
    q, s = random_8bit(4096, cols, api.DTYPE_E4M3, g)
    n = -(-rows // 4096)
    return q.repeat(n, 1)[:rows], s.view(torch.uint8).repeat(n, 1)[:rows].view(torch.float8_e8m0fnu)


def test_products_of_activations_beyond_4_gb():
    M, N, K = 530000, 64, 8208
    g = torch.Generator(device="cuda").manual_seed(10)
    a, b = big(M, K, g), random_8bit(N, K, api.DTYPE_E4M3, g, block_rows=128)
    out = run_product(AG, 1, M, N, K, api.B_NK, api.DTYPE_E4M3, [a], [b])[0]
    w = values(*b, block_rows=128)
    for rows in (slice(0, 100), slice(M - 1000, M)):
        x = values(a[0][rows], a[1][rows])
        e, s = x @ w.T, x.abs() @ w.abs().T
        assert ((out[rows].double() - e).abs() <= 2.0 ** -8 * e.abs() + K * 2.0 ** -23 * s).all()


def test_weight_gradients_from_activations_beyond_4_gb():
    M, N, K = 530000, 8, 8208
    g = torch.Generator(device="cuda").manual_seed(11)
    x = big(M, K, g)
    d = torch.zeros(M, N, device="cuda", dtype=torch.bfloat16)
    rows = [0, 1, 262144, 529999]
    for i, r in enumerate(rows):
        d[r, i] = 1      # dW's row i is that row of X
    dw = run_grad(AG, 1, M, N, K, api.DTYPE_E4M3, [d], [x], api.DTYPE_FP32)[0]
    for i, r in enumerate(rows):
        assert torch.equal(dw[i].double(), values(x[0][r:r + 1], x[1][r:r + 1])[0])
    assert (dw[4:] == 0).all()


def test_a_weight_gradient_beyond_4_gb():
    M, N, K = 3, 33024, 33296
    d, x = grad_inputs(AG, 1, M, N, K, api.DTYPE_E4M3, 12, whole=True)
    dw = run_grad(AG, 1, M, N, K, api.DTYPE_E4M3, d, x, api.DTYPE_FP32)[0]
    assert dw.numel() * 4 > 2 ** 32
    v = values(*x[0])
    for rows in (slice(0, 300), slice(N - 300, N)):
        assert torch.equal(dw[rows].double(), d[0][:, rows].double().T @ v)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_tensors_to_8_bits_beyond_4_gb(block_rows):
    M, cols = 270000, 16400
    g = torch.Generator(device="cuda").manual_seed(13)
    x = torch.randn(1024, cols, generator=g, device="cuda", dtype=torch.bfloat16).repeat(264, 1)[:M]
    q = api.make_quant(1, M, cols, block_rows=block_rows)
    data, scale = api.alloc_8bit(1, M, cols, block_rows=block_rows)
    api.compass_quantize(q, [x], data, scale)
    back = torch.empty_like(x)
    api.compass_dequantize(q, data, scale, [back])
    first = (M - 300) // 128 * 128
    for rows in (slice(0, 256), slice(first, M)):
        bits, v = kept(x[rows], api.DTYPE_E4M3, block_rows)
        at = slice(rows.start // block_rows, -(-rows.stop // block_rows))
        assert torch.equal(scale[0].view(torch.uint8)[at], bits)
        assert torch.equal(data[0][rows].double() * expand(scale[0][at], *v.shape, block_rows), v) and torch.equal(back[rows].double(), v)


def test_a_norm_in_8_bits_beyond_4_gb():
    M, H = 280000, 16400
    g = torch.Generator(device="cuda").manual_seed(14)
    x = torch.randn(1000, H, generator=g, device="cuda", dtype=torch.bfloat16).repeat(280, 1)
    n = api.make_rms_norm(1, M, H)
    y8, scale = api.alloc_8bit(1, M, H)
    api.compass_rms_norm(n, [x], None, Y8=y8, scale=scale)
    one, ones = api.alloc_8bit(1, 1000, H)
    api.compass_rms_norm(api.make_rms_norm(1, 1000, H), [x[:1000]], None, Y8=one, scale=ones)
    for i in (0, 139, 279):
        rows = slice(i * 1000, i * 1000 + 1000)
        assert torch.equal(y8[0][rows].view(torch.uint8), one[0].view(torch.uint8)) and torch.equal(scale[0][rows].view(torch.uint8), ones[0].view(torch.uint8))


# activation rows in several tiles, several shards a tile, and contractions that CTAs share
TILED = [(AG, 1, 700, 96, 4112), (AG, 16, 640, 64, 4112), (RS, 8, 600, 112, 2064)]


@pytest.mark.parametrize("layout", [api.B_NK, api.B_KN])
@pytest.mark.parametrize("op,P,M,N,K", TILED)
def test_row_tiles_read_nothing_else(op, P, M, N, K, layout):
    a, b = product_inputs(op, P, M, N, K, layout, api.DTYPE_E5M2, 8)
    want = run_product(op, P, M, N, K, layout, api.DTYPE_E5M2, a, b)
    a, b = ([(among_nan(q, 255), among_nan(s, 255)) for q, s in t] for t in (a, b))
    for x, y in zip(want, run_product(op, P, M, N, K, layout, api.DTYPE_E5M2, a, b)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("op,P,M,N,K", TILED)
def test_what_is_not_a_number_stays_in_its_row_of_a_tile(op, P, M, N, K):
    """One row of the last rank's last shard, in a value and in a scale."""
    a, b = product_inputs(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3, 9)
    clean = run_product(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3, a, b)
    a[-1][0].view(torch.uint8)[-1, 0] = NAN
    a[-1][1].view(torch.uint8)[-3, -1] = 255
    got = run_product(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3, a, b)
    for r in range(P):
        bad = torch.zeros_like(clean[r], dtype=torch.bool)
        if op == AG or r == P - 1:
            bad[[-1, -3]] = True
        assert got[r][bad].isnan().all() and torch.equal(got[r][~bad], clean[r][~bad])


@pytest.mark.parametrize("grad", [api.DTYPE_BF16, api.DTYPE_FP32])
@pytest.mark.parametrize("op,P,M,N,K", [(AG, 4, 44, 264, 400), (RS, 16, 16, 72, 272), (RS, 5, 315, 1032, 144), (AG, 1, 4100, 136, 272)])
def test_weight_gradients_of_short_shards_read_nothing_else(op, P, M, N, K, grad):
    """Shards of fewer rows than are loaded at a time, and a contraction that CTAs share."""
    d, x = grad_inputs(op, P, M, N, K, api.DTYPE_E4M3, 10)
    want = run_grad(op, P, M, N, K, api.DTYPE_E4M3, d, x, grad)
    d2, x2 = [among_nan(t, 255) for t in d], [(among_nan(q), among_nan(s, 255)) for q, s in x]
    for a, b in zip(want, run_grad(op, P, M, N, K, api.DTYPE_E4M3, d2, x2, grad)):
        assert torch.equal(a, b)


def test_shared_contractions_at_once():
    """Products and weight gradients whose CTAs wait for one another, on two streams at a time, many in flight."""
    made = []
    for seed, (op, P, M, N, K) in enumerate(TILED + [(AG, 1, 1, 4096, 4096)]):
        a, b = product_inputs(op, P, M, N, K, api.B_NK, api.DTYPE_E4M3, seed)
        pr = api.make_problem(op, P, M, N, K, dtype=api.DTYPE_E4M3)
        out = [torch.empty(M if op == AG else M // P, N, device="cuda", dtype=torch.bfloat16) for _ in range(P)]
        call = api.compass_ag_gemm_8bit if op == AG else api.compass_gemm_rs_8bit
        args = [pr, [t[0] for t in a], [t[1] for t in a], [t[0] for t in b], [t[1] for t in b], out, api.alloc_8bit_workspace(pr)]
        made.append((lambda s, call=call, args=args: call(*args, stream=s), out, args[-1]))
    for seed, (op, P, M, N, K) in enumerate([(AG, 1, 4100, 512, 512), (RS, 4, 2064, 264, 144)]):
        d, x = grad_inputs(op, P, M, N, K, api.DTYPE_E4M3, seed)
        pr = api.make_problem(op, P, M, N, K, dtype=api.DTYPE_E4M3)
        out = [torch.empty(N, K, device="cuda", dtype=torch.bfloat16) for _ in range(P)]
        args = [pr, d, [t[0] for t in x], [t[1] for t in x], out, api.alloc_8bit_workspace(pr)]
        made.append((lambda s, args=args: api.compass_weight_grad_8bit(*args, stream=s), out, args[-1]))
    for call, _, _ in made:
        call(None)
    torch.cuda.synchronize()
    want = [[t.clone() for t in out] for _, out, _ in made]
    streams = [torch.cuda.Stream() for _ in range(2)]
    half = len(made) // 2
    for turn in range(30):
        # (each call always on the same stream: its workspace and outputs are its own)
        for i in range(half):
            made[i][0](streams[0])
            made[half + (i + turn) % half][0](streams[1])
    torch.cuda.synchronize()
    for (_, out, ws), w in zip(made, want):
        assert api.compass_read_status(ws) == (api.OK, 0)
        assert all(torch.equal(a, b) for a, b in zip(out, w))
