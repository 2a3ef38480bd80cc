"""The 8-bit operators captured and replayed on new inputs, and many calls at once, every one of whose results is looked at."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from tests.eight_bit import random_8bit
from tests.test_gpu_8bit_products import AG, RS
from tests.test_gpu_8bit_products import inputs as product_inputs
from tests.test_gpu_8bit_weight_grad import inputs as grad_inputs

pytestmark = pytest.mark.gpu


def flat(*groups):
    return [t for g in groups for pair in g for t in (pair if isinstance(pair, tuple) else (pair,))]


class Call:
    """One operator's call on tensors of its own: `inputs` may be overwritten, `again` calls into other outputs."""

    def __init__(self, inputs, make_outputs, call, workspace):
        self.inputs, self.make_outputs, self.call, self.workspace = inputs, make_outputs, call, workspace
        self.outputs = make_outputs()

    def __call__(self, outputs=None, **k):
        self.call(self.outputs if outputs is None else outputs, **k)

    def bits(self, outputs=None):
        return [t.view(torch.uint8).clone() for t in (self.outputs if outputs is None else outputs)]

    def spoil(self, outputs=None):
        for t in self.outputs if outputs is None else outputs:
            t.view(torch.uint8).fill_(0xFF)       # NaN, in every type

    def check(self):
        assert self.workspace is None or api.compass_read_status(self.workspace) == (api.OK, 0)


def product(seed, op, P, M, N, K, layout=api.B_NK):
    a, b = product_inputs(op, P, M, N, K, layout, api.DTYPE_E4M3, seed)
    pr = api.make_problem(op, P, M, N, K, dtype=api.DTYPE_E4M3, b_layout=layout)
    ws = api.alloc_8bit_workspace(pr)
    call = api.compass_ag_gemm_8bit if op == AG else api.compass_gemm_rs_8bit
    parts = [t[0] for t in a], [t[1] for t in a], [t[0] for t in b], [t[1] for t in b]
    return Call(flat(a, b), lambda: [torch.empty(M if op == AG else M // P, N, device="cuda", dtype=torch.bfloat16) for _ in range(P)],
                lambda out, **k: call(pr, *parts, out, ws, **k), ws)


def gradient(seed, op, P, M, N, K, grad):
    d, x = grad_inputs(op, P, M, N, K, api.DTYPE_E4M3, seed)
    pr = api.make_problem(op, P, M, N, K, dtype=api.DTYPE_E4M3)
    ws = api.alloc_8bit_workspace(pr)
    kind = torch.float32 if grad == api.DTYPE_FP32 else torch.bfloat16
    return Call(flat(d, x), lambda: [torch.empty(N, K, device="cuda", dtype=kind) for _ in range(P)],
                lambda out, **k: api.compass_weight_grad_8bit(pr, d, [t[0] for t in x], [t[1] for t in x], out, ws, grad_dtype=grad, **k), ws)


def kept(seed, M, cols, block_rows=1, back=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = api.make_quant(1, M, cols, block_rows=block_rows)
    if back:
        x = random_8bit(M, cols, api.DTYPE_E4M3, g, block_rows=block_rows)
        return Call(list(x), lambda: [torch.empty(M, cols, device="cuda", dtype=torch.bfloat16)],
                    lambda out, **k: api.compass_dequantize(q, [x[0]], [x[1]], out, **k), None)
    x = torch.randn(M, cols, generator=g, device="cuda", dtype=torch.bfloat16)
    return Call([x], lambda: [t[0] for t in api.alloc_8bit(1, M, cols, block_rows=block_rows)],
                lambda out, **k: api.compass_quantize(q, [x], [out[0]], [out[1]], **k), None)


def norm(seed, M, H, backward=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, r, dy = (torch.randn(M, H, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    n = api.make_rms_norm(1, M, H, param_dtype=api.DTYPE_FP32)
    gamma = torch.rand(H, generator=g, device="cuda") + 0.5
    if backward:
        rstd, ws = torch.rand(M, generator=g, device="cuda") + 0.5, api.alloc_rms_norm_workspace(n)
        return Call([x, r, dy, gamma, rstd], lambda: [torch.empty_like(x), torch.empty(H, device="cuda")],
                    lambda out, **k: api.compass_rms_norm_backward(n, [dy], [x], gamma, rstd, [out[0]], out[1], ws, dsum=[r], **k), None)
    return Call([x, r, gamma], lambda: [torch.empty_like(x), torch.empty_like(x), torch.empty(M, device="cuda")] + [t[0] for t in api.alloc_8bit(1, M, H)],
                lambda out, **k: api.compass_rms_norm(n, [x], gamma, Y=[out[0]], summed=[out[1]], rstd=out[2], residual=[r], Y8=[out[3]], scale=[out[4]], **k), None)


def calls(seed):
    """Every operator, every kernel of the products and of the weight gradient."""
    return [
        product(seed, AG, 1, 1, 4096, 4096), product(seed + 1, AG, 2, 118, 1003, 2064), product(seed + 2, RS, 2, 700, 400, 1040),
        product(seed + 3, AG, 1, 256, 512, 1024, api.B_KN), product(seed + 4, RS, 8, 600, 112, 2064), product(seed + 5, AG, 3, 999, 2048, 528),
        gradient(seed + 6, AG, 2, 1500, 520, 656, api.DTYPE_BF16), gradient(seed + 7, RS, 4, 2064, 264, 144, api.DTYPE_FP32),
        gradient(seed + 8, AG, 1, 4100, 512, 512, api.DTYPE_BF16), gradient(seed + 9, AG, 1, 700, 6152, 2064, api.DTYPE_BF16),
        kept(seed + 10, 300, 528), kept(seed + 11, 300, 528, block_rows=128), kept(seed + 12, 300, 528, back=True),
        norm(seed + 13, 300, 528), norm(seed + 14, 300, 528, backward=True), norm(seed + 15, 200, 12288), norm(seed + 16, 200, 12288, backward=True),
    ]


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_captured_and_replayed_on_other_inputs():
    """The captured calls' tensors get other inputs before each replay; what comes out is what calls made at once give for them."""
    made = calls(100)
    for c in made:
        c()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in made:
            c()
    seen = [c.bits() for c in made]
    for turn in (1, 2):
        others = calls(100 + 50 * turn)
        want = []
        for c, o in zip(made, others):
            for t, u in zip(c.inputs, o.inputs):
                t.copy_(u)
            o()
            o.check()
            want.append(o.bits())
            c.spoil()
        graph.replay()
        torch.cuda.synchronize()
        for c, w, s in zip(made, want, seen):
            c.check()
            assert equal(c.bits(), w) and not equal(w, s)
        seen = want


@pytest.mark.parametrize("programs", [2, 3])
def test_calls_at_once_into_outputs_of_their_own(programs):
    """Two or three programs on a stream each, 20 rounds in flight, every round's outputs by themselves; NaN before."""
    made = [calls(300 + 100 * i) for i in range(programs)]
    want = []
    for program in made:
        for c in program:
            c.spoil()
            c()
        torch.cuda.synchronize()
        want.append([c.bits() for c in program])
    streams = [torch.cuda.Stream() for _ in made]
    rounds = [[[c.make_outputs() for c in program] for program in made] for _ in range(20)]
    for r in rounds:
        for program, outs in zip(made, r):
            for c, out in zip(program, outs):
                c.spoil(out)
    torch.cuda.synchronize()
    for turn, r in enumerate(rounds):
        order = range(len(made[0]))
        for i in order:
            for k, (program, outs) in enumerate(zip(made, r)):
                j = (i * (1 + 2 * k) + turn * k) % len(program)      # (each in another order: 17 calls, steps of 1, 3 and 5)
                program[j](outs[j], stream=streams[k])
    torch.cuda.synchronize()
    for program, w in zip(made, want):
        for c in program:
            c.check()
    for r in rounds:
        for program, outs, w in zip(made, r, want):
            for c, out, v in zip(program, outs, w):
                assert equal(c.bits(out), v)
