"""Timed cases of the operators around a tensor-parallel block: the embedding lookup, the layer norm and the loss of the
output layer, each forward and backward.

Every case runs either in its plain form (elementary torch operations in 32 bits) or, with ``own`` set, through
``paper_2609_10549_b200.api``.  Activations are [M, hidden], split by rows over P logical ranks; tables are
[vocab, hidden], split into P runs of ceil(vocab / P) rows.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one decoding step of a small batch: latency
        dict(name="embedding-step", op="embedding", way="forward", P=1, M=8, hidden=4096, vocab=32000, dtype="bf16"),
        # a long batch of two 8192-token sequences on eight ranks
        dict(name="embedding-batch", op="embedding", way="forward", P=8, M=16384, hidden=8192, vocab=128000, dtype="bf16"),
        # a short fine-tuning batch in 32 bits, odd in every size
        dict(name="embedding-grad-odd", op="embedding", way="backward", P=1, M=1001, hidden=1001, vocab=32001, dtype="fp32"),
        # the table's gradient for a training batch on eight ranks
        dict(name="embedding-grad-batch", op="embedding", way="backward", P=8, M=16384, hidden=4096, vocab=128000, dtype="bf16"),
        # one decoding step of a small batch: latency, no statistics kept
        dict(name="norm-step", op="norm", way="forward", P=1, M=8, hidden=4096, dtype="bf16", param="bf16", residual=False),
        # residual sum and norm between two blocks of a training batch
        dict(name="norm-batch", op="norm", way="forward", P=8, M=16384, hidden=8192, dtype="bf16", param="fp32", residual=True),
        # a 32-bit model with an odd hidden size
        dict(name="norm-grad-odd", op="norm", way="backward", P=1, M=4095, hidden=1001, dtype="fp32", param="fp32", residual=False),
        # training batch on eight ranks, the gradient of the residual path joined in
        dict(name="norm-grad-batch", op="norm", way="backward", P=8, M=8192, hidden=4096, dtype="bf16", param="fp32", residual=True),
        # scoring the last tokens of a few prompts
        dict(name="loss-score", op="loss", way="forward", P=1, M=16, hidden=4096, vocab=32000, ignored=0, scale=1.0, smoothing=0.0),
        # evaluation of a training batch on four ranks
        dict(name="loss-batch", op="loss", way="forward", P=4, M=8192, hidden=4096, vocab=32000, ignored=800, scale=1.0, smoothing=0.0),
        # a small model's step with label smoothing, ragged in tokens and vocabulary
        dict(name="loss-grad-odd", op="loss", way="backward", P=1, M=501, hidden=1024, vocab=50001, ignored=100, scale=0.5, smoothing=0.1),
        # a large vocabulary's training step on eight ranks
        dict(name="loss-grad-batch", op="loss", way="backward", P=8, M=8192, hidden=4096, vocab=128000, ignored=800, scale=1.0,
             smoothing=0.0),
    ]


def _between(rng, low, high):
    """Spread over the logarithm of the range."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op, way = rng.choice(("embedding", "norm", "loss")), rng.choice(("forward", "backward"))
    P = rng.choice((1, 1, 2, 4, 8))
    case = dict(op=op, way=way, P=P)
    if op == "loss":
        hidden = 8 * _between(rng, 8, 1024)
        vocab = _between(rng, 1000, 128000)
        most = min(8192, (8192 * 4096 * 128000) // (hidden * vocab))
        M = P * max(1, _between(rng, 1, max(1, most)) // P)
        return dict(case, M=M, hidden=hidden, vocab=vocab, ignored=int(M * rng.choice((0.0, 0.1, 0.5))), scale=rng.choice((1.0, 1.0, 0.5)),
                    smoothing=rng.choice((0.0, 0.0, 0.1)))
    hidden = _between(rng, 64, 8192)
    if rng.random() < 0.7:
        hidden = max(64, hidden // 64 * 64)
    M = P * max(1, _between(rng, 1, 16384) // P)
    case.update(M=M, hidden=hidden, dtype=rng.choice(("bf16", "bf16", "fp32")))
    if op == "embedding":
        return dict(case, vocab=_between(rng, 1000, 128000))
    return dict(case, param="fp32" if case["dtype"] == "fp32" else rng.choice(("bf16", "fp32")), residual=rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _shards(whole, P):
    """The ranks' runs of rows, as views: ceil(rows / P) each, the last ones shorter."""
    step = -(-whole.shape[0] // P)
    return [whole[min(r * step, whole.shape[0]):min((r + 1) * step, whole.shape[0])] for r in range(P)]


def _tokens(M, vocab, g):
    """Token ids whose frequency falls like 1 / rank, as in text."""
    u = torch.rand(M, generator=g, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1)).to(torch.int64) - 1).clamp_(0, vocab - 1)


def _lse(x, table, scale):
    """log sum exp of the scaled logits of every row: what the forward pass left."""
    parts = [(x[i:i + 1024].float() @ table.float().T).mul_(scale).logsumexp(1) for i in range(0, x.shape[0], 1024)]
    return torch.cat(parts)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = dict(case)
    P, M, H = case["P"], case["M"], case["hidden"]
    forward = case["way"] == "forward"
    if case["op"] == "embedding":
        t = DTYPES[case["dtype"]]
        V = case["vocab"]
        ids = _tokens(M, V, g)
        ids[torch.rand(M, generator=g, device="cuda") < 0.02] = -1       # padding
        s.update(ids=ids, scale=math.sqrt(H))
        if forward:
            s.update(table=(normal(V, H) * 0.02).to(t), out=torch.empty(M, H, device="cuda", dtype=t))
            names = ("table", "out")
        else:
            s.update(dout=(normal(M, H) * 1e-3).to(t), dtable=torch.empty(V, H, device="cuda", dtype=t))
            names = ("dout", "dtable")
    elif case["op"] == "norm":
        t, pt = DTYPES[case["dtype"]], DTYPES[case["param"]]
        s.update(x=(normal(M, H) + 0.5).to(t), gamma=(1 + 0.1 * normal(H)).to(pt), beta=(0.1 * normal(H)).to(pt))
        names = ("x",)
        if forward:
            s.update(y=torch.empty(M, H, device="cuda", dtype=t))
            names += ("y",)
            if case["residual"]:
                s.update(residual=normal(M, H).to(t), summed=torch.empty(M, H, device="cuda", dtype=t),
                         mean=torch.empty(M, device="cuda"), rstd=torch.empty(M, device="cuda"))
                names += ("residual", "summed")
        else:
            x = s["x"].float()
            mean = x.mean(1)
            s.update(mean=mean, rstd=((x - mean[:, None]).square().mean(1) + 1e-5).rsqrt(), dy=(normal(M, H) * 1e-2).to(t),
                     dx=torch.empty(M, H, device="cuda", dtype=t), dgamma=torch.empty(H, device="cuda", dtype=pt),
                     dbeta=torch.empty(H, device="cuda", dtype=pt))
            names += ("dy", "dx")
            if case["residual"]:
                s.update(dsum=(normal(M, H) * 1e-2).to(t))
                names += ("dsum",)
    else:
        V = case["vocab"]
        table = (normal(V, H) * (1.3 / math.sqrt(H))).to(torch.bfloat16)
        targets = _tokens(M, V, g)
        # hidden states as a trained model has them: some targets are almost certain, some are not expected at all
        toward = table[targets].float()
        x = normal(M, H) + toward * (torch.rand(M, 1, generator=g, device="cuda") * 9)
        x = x.to(torch.bfloat16)
        targets[torch.randperm(M, generator=g, device="cuda")[:case["ignored"]]] = -100     # prompt and padding
        s.update(x=x, table=table, targets=targets)
        names = ("x", "table")
        if forward:
            s.update(loss=torch.empty(M, device="cuda"), lse=torch.empty(M, device="cuda"))
        else:
            valid = targets >= 0
            s.update(lse=_lse(x, table, case["scale"]), dloss=valid.float() / valid.sum().clamp(min=1),
                     dx=torch.empty_like(x), dtable=torch.empty_like(table))
            names += ("dx", "dtable")
    for n in names:
        s[n + "_shards"] = _shards(s[n], P)
    s["plan"] = {}
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------


def _plain(s):
    if s["op"] == "embedding":
        ids, valid = s["ids"], s["ids"] >= 0
        if s["way"] == "forward":
            rows = s["table"][ids.clamp(min=0)].float() * s["scale"]
            return {"out": (rows * valid[:, None]).to(s["table"].dtype)}
        total = torch.zeros(s["vocab"], s["hidden"], device="cuda")
        total.index_add_(0, ids[valid], s["dout"][valid].float())
        return {"dtable": (total * s["scale"]).to(s["dout"].dtype)}
    if s["op"] == "norm":
        g = s["gamma"].float()
        if s["way"] == "forward":
            h = s["x"].float()
            if s["residual"] is not False:
                h = (h + s["residual"].float()).to(s["x"].dtype)
                summed, h = h, h.float()
            mean = h.mean(1)
            c = h - mean[:, None]
            rstd = torch.rsqrt((c * c).mean(1) + 1e-5)
            y = (c * rstd[:, None] * g + s["beta"].float()).to(s["x"].dtype)
            return {"y": y} if s["residual"] is False else {"y": y, "summed": summed, "mean": mean, "rstd": rstd}
        dy = s["dy"].float()
        xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        gd = dy * g
        dx = (gd - gd.mean(1, keepdim=True) - xh * (gd * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
        if s["residual"] is not False:
            dx = dx + s["dsum"].float()
        return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xh).sum(0).to(s["gamma"].dtype), "dbeta": dy.sum(0).to(s["gamma"].dtype)}
    valid = s["targets"] >= 0
    at = s["targets"].clamp(min=0)[:, None]
    x, w = s["x"].float(), s["table"].float()
    z = (x @ w.T).mul_(s["scale"])
    e, V = s["smoothing"], s["vocab"]
    if s["way"] == "forward":
        top = z.max(1, keepdim=True).values
        lse = top[:, 0] + torch.log(torch.exp(z - top).sum(1))
        loss = lse - (1 - e) * z.gather(1, at)[:, 0]
        if e:
            loss = loss - e / V * z.sum(1)
        zero = torch.zeros_like(lse)
        return {"loss": torch.where(valid, loss, zero), "lse": torch.where(valid, lse, zero)}
    d = torch.exp_(z.sub_(s["lse"][:, None]))
    if e:
        d.sub_(e / V)
    d.scatter_add_(1, at, torch.full_like(d[:, :1], e - 1))
    d.mul_((s["dloss"] * valid * s["scale"])[:, None])
    return {"dx": (d @ w).to(torch.bfloat16), "dtable": (d.T @ x).to(torch.bfloat16)}


# ---- the framework's operators --------------------------------------------------------------------------------------


def _own(s):
    from paper_2609_10549_b200 import api

    plan = s["plan"]
    if s["op"] == "embedding":
        if not plan:
            plan["op"] = api.make_embedding(s["P"], s["M"], s["hidden"], s["vocab"], scale=s["scale"],
                                            dtype=api.DTYPE_BF16 if s["dtype"] == "bf16" else api.DTYPE_FP32)
            if s["way"] == "backward":
                plan["ws"] = api.alloc_embedding_workspace(plan["op"])
        if s["way"] == "forward":
            api.compass_embedding(plan["op"], s["ids"], s["table_shards"], s["out_shards"])
            return {"out": s["out"]}
        api.compass_embedding_backward(plan["op"], s["ids"], s["dout_shards"], s["dtable_shards"], plan["ws"])
        return {"dtable": s["dtable"]}
    if s["op"] == "norm":
        if not plan:
            kind = {"bf16": api.DTYPE_BF16, "fp32": api.DTYPE_FP32}
            plan["op"] = api.make_layer_norm(s["P"], s["M"], s["hidden"], eps=1e-5, dtype=kind[s["dtype"]], param_dtype=kind[s["param"]])
            if s["way"] == "backward":
                plan["ws"] = api.alloc_layer_norm_workspace(plan["op"])
        if s["way"] == "forward":
            if s["residual"] is False:
                api.compass_layer_norm(plan["op"], s["x_shards"], s["gamma"], s["beta"], s["y_shards"])
                return {"y": s["y"]}
            api.compass_layer_norm(plan["op"], s["x_shards"], s["gamma"], s["beta"], s["y_shards"], mean=s["mean"], rstd=s["rstd"],
                                   residual=s["residual_shards"], summed=s["summed_shards"])
            return {"y": s["y"], "summed": s["summed"], "mean": s["mean"], "rstd": s["rstd"]}
        api.compass_layer_norm_backward(plan["op"], s["dy_shards"], s["x_shards"], s["gamma"], s["mean"], s["rstd"], s["dx_shards"],
                                        s["dgamma"], s["dbeta"], plan["ws"], dsum=s.get("dsum_shards"))
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if not plan:
        plan["op"] = api.make_head(s["P"], s["M"], s["hidden"], s["vocab"], logit_scale=s["scale"], label_smoothing=s["smoothing"])
        plan["ws"] = api.alloc_head_workspace(plan["op"], backward=s["way"] == "backward")
    if s["way"] == "forward":
        api.compass_head_loss(plan["op"], s["x_shards"], s["table_shards"], s["targets"], s["loss"], s["lse"], plan["ws"])
        return {"loss": s["loss"], "lse": s["lse"]}
    api.compass_head_loss_backward(plan["op"], s["x_shards"], s["table_shards"], s["targets"], s["lse"], s["dloss"], s["dx_shards"],
                                   s["dtable_shards"], plan["ws"])
    return {"dx": s["dx"], "dtable": s["dtable"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    M, H = case["M"], case["hidden"]
    forward = case["way"] == "forward"
    size = 4 if case.get("dtype") == "fp32" else 2
    if case["op"] == "embedding":
        return {"bytes": 8 * M + size * M * H + size * H * (M if forward else case["vocab"]), "flops": M * H}
    if case["op"] == "norm":
        params = 4 if case["param"] == "fp32" else 2
        tensors = (2 + 2 * case["residual"]) if forward else (3 + case["residual"])
        stats = 8 * M if not forward or case["residual"] else 0
        return {"bytes": tensors * size * M * H + stats + (2 if forward else 3) * params * H, "flops": (8 if forward else 14) * M * H}
    rows, V = M - case["ignored"], case["vocab"]
    if forward:
        return {"bytes": 2 * (rows + V) * H + 16 * M, "flops": 2 * rows * H * V}
    return {"bytes": 4 * (rows + V) * H + 16 * M, "flops": 6 * rows * H * V}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    M, H = case["M"], case["hidden"]
    if case["op"] == "embedding":
        ids = s["ids"].cpu()
        keep = (ids >= 0).nonzero()[:, 0]
        if case["way"] == "forward":
            out = torch.zeros(M, H, dtype=torch.float64)
            out[keep] = s["table"][ids[keep].cuda()].double().cpu() * s["scale"]
            return {"out": out}
        # the tokens' gradients in the order of their ids, each id's run summed
        order = keep[torch.argsort(ids[keep], stable=True)]
        found, counts = torch.unique_consecutive(ids[order], return_counts=True)
        grad = torch.zeros(case["vocab"], H, dtype=torch.float64, device="cuda")
        d = s["dout"][order.cuda()].double()
        grad[found.cuda()] = torch.segment_reduce(d, "sum", lengths=counts.cuda(), axis=0) * s["scale"]
        return {"dtable": grad}
    if case["op"] == "norm":
        h = s["x"].double()
        if case["way"] == "forward":
            kept = None
            if case["residual"]:
                # the sum is stored in the activations' type, and what is stored is normalised
                kept = h + s["residual"].double()
                h = (s["x"].float() + s["residual"].float()).to(s["x"].dtype).double()
            var, mean = torch.var_mean(h, 1, correction=0, keepdim=True)
            y = torch.addcmul(s["beta"].double(), (h - mean) / torch.sqrt(var + 1e-5), s["gamma"].double())
            if kept is None:
                return {"y": y}
            return {"y": y, "summed": kept, "mean": mean[:, 0], "rstd": 1 / torch.sqrt(var[:, 0] + 1e-5)}
        # by the Jacobian's rows: d xh / d x = rstd (I - 1/n - xh xh^T / n), for the statistics that were handed in
        r = s["rstd"].double()[:, None]
        xh = torch.sub(h, s["mean"].double()[:, None]) * r
        up = s["dy"].double()
        v = up * s["gamma"].double()
        dx = r * (v - (v.sum(1, keepdim=True) + xh * torch.einsum("ij,ij->i", v, xh)[:, None]) / H)
        if case["residual"]:
            dx += s["dsum"].double()
        return {"dx": dx, "dgamma": torch.einsum("ij,ij->j", up, xh), "dbeta": torch.einsum("ij->j", up)}
    V, e, c = case["vocab"], case["smoothing"], case["scale"]
    w = s["table"].double()
    rows = (s["targets"] >= 0).nonzero()[:, 0]
    loss, lse = (torch.zeros(M, dtype=torch.float64, device="cuda") for _ in range(2))
    if case["way"] == "backward":
        dx, dw = torch.zeros(M, H, dtype=torch.float64, device="cuda"), torch.zeros(V, H, dtype=torch.float64, device="cuda")
    for part in rows.split(1024):
        x = s["x"][part].double()
        y = torch.nn.functional.one_hot(s["targets"][part], V) if V * part.numel() < 1 << 22 else None
        z = torch.mm(x, w.t()) * c
        if case["way"] == "forward":
            lse[part] = torch.logsumexp(z, 1)
            picked = (z * y).sum(1) if y is not None else torch.take_along_dim(z, s["targets"][part][:, None], 1).squeeze(1)
            loss[part] = (1 - e) * (lse[part] - picked) + e * (lse[part] - z.mean(1))
        else:
            p = torch.exp(z - s["lse"][part].double()[:, None]) - e / V
            p[torch.arange(part.numel(), device="cuda"), s["targets"][part]] -= 1 - e
            p *= s["dloss"][part].double()[:, None] * c
            dx[part] = torch.mm(p, w)
            dw += torch.mm(p.t(), x)
    return {"loss": loss, "lse": lse} if case["way"] == "forward" else {"dx": dx, "dtable": dw}
