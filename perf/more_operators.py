"""Timed cases of a linear block that computes and keeps its activations in 8 bits: the root-mean-square norm (with the
residual sum, its output in 8 bits), activations kept in 8 bits and restored, the tensor-parallel products of 8-bit
operands, and the weights' gradient from activations kept in 8 bits.

Every case runs either in its plain form (elementary torch operations in 32 bits) or, with ``own`` set, through
``paper_2609_10549_b200.api``.  An 8-bit tensor is values in E4M3 or E5M2 with a power of two for each run of 128 columns
(activations) or each 128 x 128 block (weights), stored as its exponent (E8M0).  Activations are split by rows over P
logical ranks, weights are one [N, K] tensor per rank.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}


def listed():
    return [
        # the norm before the next token's projection: latency
        dict(name="norm8-token", op="norm", way="forward", P=1, M=1, hidden=4096, dtype="bf16", param="bf16", residual=True, out="e4m3"),
        # residual sum and norm between two blocks of a training batch, for 8-bit products
        dict(name="norm8-batch", op="norm", way="forward", P=8, M=16384, hidden=8192, dtype="bf16", param="fp32", residual=True, out="e4m3"),
        # a 32-bit model with an odd hidden size
        dict(name="rms-grad-odd", op="norm", way="backward", P=1, M=4095, hidden=1001, dtype="fp32", param="fp32", residual=False, out="fp32"),
        # training batch on eight ranks, the gradient of the residual path joined in
        dict(name="rms-grad-batch", op="norm", way="backward", P=8, M=8192, hidden=4096, dtype="bf16", param="fp32", residual=True, out="bf16"),
        # a small 32-bit activation kept for the backward pass
        dict(name="keep8-odd", op="keep", P=1, M=1003, cols=1040, dtype="fp32", format="e5m2"),
        # a training batch's activations kept and restored
        dict(name="keep8-batch", op="keep", P=4, M=16384, cols=8192, dtype="bf16", format="e4m3"),
        # a projection of the next token: the weights' bytes
        dict(name="product8-token", op="product", kind="ag", layout="nk", P=1, M=1, N=4096, K=4096, format="e4m3"),
        # a few prompts' last tokens, ragged in every size
        dict(name="product8-few-odd", op="product", kind="ag", layout="nk", P=2, M=118, N=5003, K=2064, format="e4m3"),
        # first product of a feed-forward block of a training batch on eight ranks
        dict(name="product8-batch", op="product", kind="ag", layout="nk", P=8, M=8192, N=1376, K=4096, format="e4m3"),
        # its data gradient: summed over four ranks, on the stored weights
        dict(name="product8-grad-batch", op="product", kind="rs", layout="kn", P=4, M=8192, N=4096, K=2752, format="e5m2"),
        # a small model's weight gradient in 32 bits, ragged
        dict(name="weight-grad8-odd", op="weight", kind="ag", P=1, M=501, N=1000, K=2064, format="e4m3", grad="fp32"),
        # weight gradient of a feed-forward block of a training batch on four ranks
        dict(name="weight-grad8-batch", op="weight", kind="ag", P=4, M=8192, N=2752, K=4096, format="e4m3", grad="bf16"),
    ]


def _between(rng, low, high):
    """Spread over the logarithm of the range."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("norm", "keep", "product", "product", "weight"))
    P = rng.choice((1, 1, 2, 4, 8))
    if op == "norm":
        way, dtype = rng.choice(("forward", "forward", "backward")), rng.choice(("bf16", "bf16", "fp32"))
        out = dtype if way == "backward" or rng.random() < 0.3 else rng.choice(("e4m3", "e4m3", "e5m2"))
        hidden = _between(rng, 64, 8192)
        if out in FORMATS or rng.random() < 0.7:
            hidden = max(64, hidden // 16 * 16)
        M = P * max(1, _between(rng, 1, 16384) // P)
        return dict(op=op, way=way, P=P, M=M, hidden=hidden, dtype=dtype, param="fp32" if dtype == "fp32" else rng.choice(("bf16", "fp32")),
                    residual=rng.random() < 0.6, out=out)
    if op == "keep":
        return dict(op=op, P=P, M=P * max(1, _between(rng, 1, 16384) // P), cols=16 * _between(rng, 4, 512), dtype=rng.choice(("bf16", "bf16", "fp32")),
                    format=rng.choice(("e4m3", "e4m3", "e5m2")))
    K, M = 16 * _between(rng, 4, 512), P * max(1, _between(rng, 1, 8192) // P)
    kind = rng.choice(("ag", "rs"))
    most = max(8, min(8192, (8192 * 4096 * 2752 * 4) // (P * M * K)))        # as many operations as the largest listed case
    N = _between(rng, 64, max(64, most))
    if op == "product":
        layout = rng.choice(("nk", "nk", "kn"))
        return dict(op=op, kind=kind, layout=layout, P=P, M=M, N=max(64, N // 16 * 16) if layout == "kn" else N, K=K,
                    format=rng.choice(("e4m3", "e4m3", "e5m2")))
    return dict(op=op, kind=kind, P=P, M=M, N=max(64, N // 8 * 8), K=K, format=rng.choice(("e4m3", "e4m3", "e5m2")), grad=rng.choice(("bf16", "bf16", "fp32")))


# ---- 8-bit tensors, plain ---------------------------------------------------------------------------------------------


def _blocks(n):
    return -(-n // 128)


def _runs(x, fill=0):
    """[rows, cols] as [rows, ceil(cols / 128), 128], filled up."""
    rows, cols = x.shape
    return torch.nn.functional.pad(x, (0, _blocks(cols) * 128 - cols), value=fill).view(rows, -1, 128)


def _exponent(top, format):
    """Smallest e >= -127 with top <= largest number of the format * 2^e."""
    mantissa, e = torch.frexp(top / LARGEST[format])            # top / largest = mantissa * 2^e, mantissa in [0.5, 1)
    e = torch.where(mantissa > 0.5, e, e - 1)
    return torch.where(top > 0, e, torch.full_like(e, -127)).clamp(min=-127)


def _store(x, format, rows_too=False):
    """Values and E8M0 scales of a matrix: per run of 128 columns, or per 128 x 128 block."""
    r = _runs(x.float())
    top = r.abs().amax(2)
    if rows_too:
        n = top.shape[0]
        top = torch.nn.functional.pad(top, (0, 0, 0, _blocks(n) * 128 - n)).view(-1, 128, top.shape[1]).amax(1)
    e = _exponent(top, format)
    per_row = e.repeat_interleave(128, 0)[:x.shape[0]] if rows_too else e
    q = torch.ldexp(r, -per_row[:, :, None]).view(x.shape[0], -1)[:, :x.shape[1]].contiguous().to(FORMATS[format])
    return q, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _values(q, scale, rows_too=False):
    """What an 8-bit tensor stands for, in 32 bits."""
    f = torch.exp2(scale.view(torch.uint8).float() - 127)
    if rows_too:
        f = f.repeat_interleave(128, 0)[:q.shape[0]]
    return (_runs(q.float()) * f[:, :, None]).view(q.shape[0], -1)[:, :q.shape[1]]


# ---- inputs -----------------------------------------------------------------------------------------------------------


def _shards(whole, P):
    """The ranks' equal runs of rows, as views."""
    return list(whole.split(whole.shape[0] // P))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731

    def activations(rows, cols):
        """Some channels are much larger than the others, some rows too."""
        x = normal(rows, cols)
        x *= torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, 20.0, 1.0)
        return x.mul_(torch.exp(0.5 * normal(rows, 1)))

    s = dict(case)
    P, M = case["P"], case["M"]
    if case["op"] == "norm":
        H, t, pt = case["hidden"], DTYPES[case["dtype"]], DTYPES[case["param"]]
        s.update(x=activations(M, H).to(t), gamma=(1 + 0.1 * normal(H)).to(pt))
        names = ["x"]
        if case["way"] == "forward":
            # what is kept in 8 bits is restored in BF16, which holds every such value
            s.update(rstd=torch.empty(M, device="cuda"), y=torch.empty(M, H, device="cuda", dtype=torch.bfloat16 if case["out"] in FORMATS else t))
            names += ["y"]
            if case["residual"]:
                s.update(residual=normal(M, H).to(t), summed=torch.empty(M, H, device="cuda", dtype=t))
                names += ["residual", "summed"]
            if case["out"] in FORMATS:
                s.update(q=torch.empty(M, H, device="cuda", dtype=FORMATS[case["out"]]),
                         scale=torch.empty(M, _blocks(H), device="cuda", dtype=torch.float8_e8m0fnu))
                names += ["q", "scale"]
        else:
            s.update(rstd=(s["x"].double().square().mean(1) + 1e-5).rsqrt().float(), dy=(normal(M, H) * 1e-2).to(t),
                     dx=torch.empty(M, H, device="cuda", dtype=t), dgamma=torch.empty(H, device="cuda", dtype=pt))
            names += ["dy", "dx"]
            if case["residual"]:
                s.update(dsum=(normal(M, H) * 1e-2).to(t))
                names += ["dsum"]
    elif case["op"] == "keep":
        t = DTYPES[case["dtype"]]
        s.update(x=activations(M, case["cols"]).to(t), q=torch.empty(M, case["cols"], device="cuda", dtype=FORMATS[case["format"]]),
                 scale=torch.empty(M, _blocks(case["cols"]), device="cuda", dtype=torch.float8_e8m0fnu), y=torch.empty(M, case["cols"], device="cuda", dtype=t))
        names = ["x", "q", "scale", "y"]
    else:
        N, K = case["N"], case["K"]
        gathered = case["kind"] == "ag"
        # the 8-bit activations: one matrix in row shards, or one per rank
        x = [_store(activations(M, K).to(torch.bfloat16), case["format"]) for _ in range(1 if gathered else P)]
        s["x8"], s["x_scale"] = ([_shards(a, P) for a in x[0]] if gathered else zip(*x))
        s["x8"], s["x_scale"] = list(s["x8"]), list(s["x_scale"])
        if case["op"] == "product":
            shape = (N, K) if case["layout"] == "nk" else (K, N)
            w = [_store(normal(*shape) / math.sqrt(K * (1 if gathered else P)), "e4m3", True) for _ in range(P)]
            s.update(w8=[a[0] for a in w], w_scale=[a[1] for a in w],
                     out=[torch.empty(M if gathered else M // P, N, device="cuda", dtype=torch.bfloat16) for _ in range(P)])
        else:
            # the products' outputs and their gradients: one per rank, or one in row shards
            dy = [(normal(M, N) * 1e-2).to(torch.bfloat16) for _ in range(P if gathered else 1)]
            s.update(dy=dy if gathered else _shards(dy[0], P), dw=[torch.empty(N, K, device="cuda", dtype=DTYPES[case["grad"]]) for _ in range(P)])
        names = []
    for n in names:
        s[n + "_shards"] = _shards(s[n], P)
    s["plan"] = {}
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------


def _plain(s):
    if s["op"] == "keep":
        return {"values": _values(*_store(s["x"], s["format"])).to(s["x"].dtype)}
    if s["op"] == "norm":
        t, g, n = s["x"].dtype, s["gamma"].float(), s["hidden"]
        if s["way"] == "forward":
            h, got = s["x"].float(), {}
            if s["residual"] is not False:
                got["summed"] = (h + s["residual"].float()).to(t)
                h = got["summed"].float()
            got["rstd"] = torch.rsqrt((h * h).sum(1) / n + 1e-5)
            y = h * got["rstd"][:, None] * g
            got["y"] = (_values(*_store(y, s["out"])) if s["out"] in FORMATS else y).to(s["y"].dtype)
            return got
        dy, r = s["dy"].float(), s["rstd"][:, None]
        xh, gd = s["x"].float() * r, dy * g
        dx = (gd - xh * ((gd * xh).sum(1, keepdim=True) / n)) * r
        if s["residual"] is not False:
            dx = dx + s["dsum"].float()
        return {"dx": dx.to(t), "dgamma": (dy * xh).sum(0).to(s["gamma"].dtype)}
    x = [_values(q, e) for q, e in zip(s["x8"], s["x_scale"])]
    ag = s["kind"] == "ag"
    if ag:
        x = [torch.cat(x)] * s["P"]
    if s["op"] == "weight":
        dy = s["dy"] if ag else [torch.cat(s["dy"])] * s["P"]
        return {"dw": [(d.float().T @ a).to(s["dw"][0].dtype) for d, a in zip(dy, x)]}
    w = [_values(q, e, True) for q, e in zip(s["w8"], s["w_scale"])]
    y = [a @ (b.T if s["layout"] == "nk" else b) for a, b in zip(x, w)]
    if not ag:
        y = torch.stack(y).sum(0).split(s["M"] // s["P"])
    return {"out": [a.to(torch.bfloat16) for a in y]}


# ---- the framework's operators ----------------------------------------------------------------------------------------


def _own(s):
    from paper_2609_10549_b200 import api

    plan, P, M = s["plan"], s["P"], s["M"]
    kinds = {"bf16": api.DTYPE_BF16, "fp32": api.DTYPE_FP32, "e4m3": api.DTYPE_E4M3, "e5m2": api.DTYPE_E5M2}
    if s["op"] == "keep":
        if not plan:
            plan["op"] = api.make_quant(P, M, s["cols"], dtype=kinds[s["dtype"]], format=kinds[s["format"]])
        api.compass_quantize(plan["op"], s["x_shards"], s["q_shards"], s["scale_shards"])
        api.compass_dequantize(plan["op"], s["q_shards"], s["scale_shards"], s["y_shards"])
        return {"values": s["y"]}
    if s["op"] == "norm":
        if not plan:
            plan["op"] = api.make_rms_norm(P, M, s["hidden"], eps=1e-5, dtype=kinds[s["dtype"]], param_dtype=kinds[s["param"]])
            if s["way"] == "backward":
                plan["ws"] = api.alloc_rms_norm_workspace(plan["op"])
            if s["out"] in FORMATS:
                plan["quant"] = api.make_quant(P, M, s["hidden"], format=kinds[s["out"]])
        if s["way"] == "forward":
            more = {} if s["residual"] is False else dict(residual=s["residual_shards"], summed=s["summed_shards"])
            got = {} if s["residual"] is False else {"summed": s["summed"]}
            if s["out"] in FORMATS:
                api.compass_rms_norm(plan["op"], s["x_shards"], s["gamma"], rstd=s["rstd"], Y8=s["q_shards"], scale=s["scale_shards"],
                                     format=kinds[s["out"]], **more)
                api.compass_dequantize(plan["quant"], s["q_shards"], s["scale_shards"], s["y_shards"])
            else:
                api.compass_rms_norm(plan["op"], s["x_shards"], s["gamma"], Y=s["y_shards"], rstd=s["rstd"], **more)
            return dict(got, rstd=s["rstd"], y=s["y"])
        api.compass_rms_norm_backward(plan["op"], s["dy_shards"], s["x_shards"], s["gamma"], s["rstd"], s["dx_shards"], s["dgamma"], plan["ws"],
                                      dsum=s.get("dsum_shards"))
        return {"dx": s["dx"], "dgamma": s["dgamma"]}
    ag = s["kind"] == "ag"
    if not plan:
        plan["op"] = api.make_problem(api.OP_AG_GEMM if ag else api.OP_GEMM_RS, P, M, s["N"], s["K"], dtype=kinds[s["format"]],
                                      b_layout=api.B_KN if s.get("layout") == "kn" else api.B_NK)
        plan["ws"] = api.alloc_8bit_workspace(plan["op"])
    if s["op"] == "weight":
        api.compass_weight_grad_8bit(plan["op"], s["dy"], s["x8"], s["x_scale"], s["dw"], plan["ws"], grad_dtype=kinds[s["grad"]])
        return {"dw": s["dw"]}
    call = api.compass_ag_gemm_8bit if ag else api.compass_gemm_rs_8bit
    call(plan["op"], s["x8"], s["x_scale"], s["w8"], s["w_scale"], s["out"], plan["ws"])
    return {"out": s["out"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------


def work(case):
    P, M = case["P"], case["M"]
    if case["op"] == "keep":
        size = 4 if case["dtype"] == "fp32" else 2
        # written in 8 bits, read again and restored
        return {"bytes": M * case["cols"] * (2 * size + 2) + 2 * M * _blocks(case["cols"]), "flops": 3 * M * case["cols"]}
    if case["op"] == "norm":
        H, size = case["hidden"], 4 if case["dtype"] == "fp32" else 2
        params = 4 if case["param"] == "fp32" else 2
        if case["way"] == "backward":
            return {"bytes": (3 + case["residual"]) * size * M * H + 4 * M + 2 * params * H, "flops": 10 * M * H}
        kept = 2 * M * H + 2 * M * _blocks(H) if case["out"] in FORMATS else 0      # written in 8 bits and read again
        return {"bytes": (2 + 2 * case["residual"]) * size * M * H + kept + 4 * M + params * H, "flops": 6 * M * H}
    N, K, ag = case["N"], case["K"], case["kind"] == "ag"
    x8 = (1 if ag else P) * M * (K + _blocks(K))
    if case["op"] == "weight":
        return {"bytes": x8 + 2 * (P if ag else 1) * M * N + P * N * K * (4 if case["grad"] == "fp32" else 2), "flops": 2 * P * M * N * K}
    return {"bytes": x8 + P * (N * K + _blocks(N) * _blocks(K)) + 2 * (P if ag else 1) * M * N, "flops": 2 * P * M * N * K}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------


def _kept(v, format):
    """The value that each element of a matrix in 64 bits is kept as: a multiple of the format's spacing at its size."""
    bits, low, top = {"e4m3": (3, -6, 448.0), "e5m2": (2, -14, 57344.0)}[format]
    rows, cols = v.shape
    out = torch.empty_like(v)
    for c in range(0, cols, 128):
        part = v[:, c:c + 128]
        need = torch.ceil(torch.log2(part.abs().amax(1, keepdim=True) / top))
        # (the logarithm may be off by a rounding: settled by the definition)
        largest = part.abs().amax(1, keepdim=True)
        need = need - (largest <= top * torch.exp2(need - 1)).double()
        need = (need + (largest > top * torch.exp2(need)).double()).clamp(min=-127)
        unit = part / torch.exp2(need)
        size = torch.floor(torch.log2(unit.abs().clamp(min=2.0 ** low)))
        size = size - (torch.exp2(size) > unit.abs().clamp(min=2.0 ** low)).double()
        step = torch.exp2(size - bits)
        out[:, c:c + 128] = torch.round(unit / step) * step * torch.exp2(need)
    return out


def _double(q, e, square=False):
    """An 8-bit tensor's values in 64 bits."""
    column = torch.arange(q.shape[1], device="cuda") // 128
    row = torch.arange(q.shape[0], device="cuda") // (128 if square else 1)
    return q.double() * torch.pow(2.0, e.view(torch.uint8).double() - 127.0)[row][:, column]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "keep":
        return {"values": _kept(s["x"].double(), case["format"])}
    if case["op"] == "norm":
        n, g = case["hidden"], s["gamma"].double()
        if case["way"] == "forward":
            h, got = s["x"].double(), {}
            if case["residual"]:
                got["summed"] = h + s["residual"].double()
                # the sum is stored in the activations' type, and what is stored is normalised
                h = (s["x"].float() + s["residual"].float()).to(s["x"].dtype).double()
            got["rstd"] = 1 / torch.sqrt(torch.einsum("ij,ij->i", h, h) / n + 1e-5)
            y = torch.einsum("ij,i,j->ij", h, got["rstd"], g)
            got["y"] = _kept(y, case["out"]) if case["out"] in FORMATS else y
            return got
        # by the Jacobian's rows: d xh / d x = rstd (I - xh xh^T / n), for the statistics that were handed in
        r, up = s["rstd"].double()[:, None], s["dy"].double()
        xh, v = s["x"].double() * r, up * g
        dx = r * (v - xh * torch.einsum("ij,ij->i", v, xh)[:, None] / n)
        if case["residual"]:
            dx += s["dsum"].double()
        return {"dx": dx, "dgamma": torch.einsum("ij,ij->j", up, xh)}
    P, ag = case["P"], case["kind"] == "ag"
    if case["op"] == "weight":
        dw = []
        for r in range(P):
            total = torch.zeros(case["N"], case["K"], dtype=torch.float64, device="cuda")
            for c in range(P):      # by the ranks' rows
                rows = slice(c * (case["M"] // P), (c + 1) * (case["M"] // P))
                a = _double(s["x8"][c], s["x_scale"][c]) if ag else _double(s["x8"][r], s["x_scale"][r])[rows]
                d = s["dy"][r][rows] if ag else s["dy"][c]
                total.addmm_(d.double().t(), a)
            dw.append(total)
        return {"dw": dw}
    out = []
    for r in range(P):
        parts = []
        for q in range(P):
            # the gathered rows of rank q through rank r's weights, or rank r's rows of rank q's partial product
            step = case["M"] // P
            a = _double(s["x8"][q], s["x_scale"][q]) if ag else _double(s["x8"][q][r * step:(r + 1) * step], s["x_scale"][q][r * step:(r + 1) * step])
            w = _double(s["w8"][r if ag else q], s["w_scale"][r if ag else q], True)
            parts.append(torch.mm(a, w.t() if case["layout"] == "nk" else w))
        out.append(torch.cat(parts) if ag else torch.stack(parts).sum(0))
    return {"out": out}
