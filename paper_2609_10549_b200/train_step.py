"""A tied-embedding language model on the library's operators, one training step at a time.

    python -m paper_2609_10549_b200.train_step [--products bf16|8bit] [--P 4] [--tokens 4096] [--hidden 1024] [--ffn 512] [--vocab 32000]
                                               [--layers 2] [--steps 20]

Embedding -> layers of (norm -> tensor-parallel MLP block -> residual) -> norm -> cross entropy of the output layer, whose
table is the embedding's.  Activations are split by rows over P logical ranks, the table by vocabulary rows, everything in
BF16 with norms in FP32.  torch supplies memory and the optimiser.

bf16: layer norms, MLP blocks in BF16.  Trained are the table and the norms; the MLP blocks' weights stay as they are.
8bit: root-mean-square norms; the MLP blocks' products, forward and of the data gradients, are of 8-bit operands, the
activations are kept in 8 bits alone, and the weight gradients come from those.  Everything is trained; the weights are
brought to 8 bits from BF16 at every step, whose blocks' scales serve both directions.
"""
from __future__ import annotations

import argparse
from typing import List

from . import api


class TiedModel:
    """Weights, buffers and workspaces of the model; `step` runs forward, backward and update."""

    def __init__(self, P: int, tokens: int, hidden: int, ffn: int, vocab: int, layers: int, seed: int = 0, device: str = "cuda"):
        import torch
        self.torch, self.P, self.M, self.H, self.V, self.layers = torch, P, tokens, hidden, vocab, layers
        g = torch.Generator(device=device).manual_seed(seed)
        normal = lambda scale, *shape: (torch.randn(*shape, generator=g, device=device) * scale).bfloat16()  # noqa: E731
        rows = lambda: [torch.empty(tokens // P, hidden, device=device, dtype=torch.bfloat16) for _ in range(P)]  # noqa: E731
        vector = lambda n: torch.empty(n, device=device)  # noqa: E731
        self.table = [normal(0.02, api.vocab_shard_rows(vocab, P, r), hidden) for r in range(P)]
        self.w0 = [[normal(hidden ** -0.5, ffn, hidden) for _ in range(P)] for _ in range(layers)]
        self.w1 = [[normal(0.5 * (P * ffn) ** -0.5, hidden, ffn) for _ in range(P)] for _ in range(layers)]
        self.gamma = [torch.ones(hidden, device=device) for _ in range(layers + 1)]
        self.beta = [torch.zeros(hidden, device=device) for _ in range(layers + 1)]

        # the embedding's gradient is added to what the output layer leaves in the same table
        self.embed = api.make_embedding(P, tokens, hidden, vocab, scale=hidden ** 0.5, accumulate=True)
        self.norm = api.make_layer_norm(P, tokens, hidden, param_dtype=api.DTYPE_FP32)
        self.head = api.make_head(P, tokens, hidden, vocab)
        self.mlp = api.make_mlp(P, tokens, hidden, ffn)
        self.mlp_back = api.make_mlp(P, tokens, hidden, ffn, b_layout=api.B_KN)
        self.ws_embed = api.alloc_embedding_workspace(self.embed, device)
        self.ws_norm = api.alloc_layer_norm_workspace(self.norm, device)
        self.ws_head = api.alloc_head_workspace(self.head, device=device)
        self.ws_head_back = api.alloc_head_workspace(self.head, backward=True, device=device)
        self.ws_mlp = api.alloc_mlp_workspace(self.mlp, device)
        self.ws_mlp_back = api.alloc_mlp_workspace(self.mlp_back, device)

        self.h = [rows() for _ in range(layers + 1)]              # the residual stream, before each norm
        self.y = [rows() for _ in range(layers + 1)]              # after it
        self.out = [rows() for _ in range(layers)]                # of the MLP blocks
        self.mid = [[torch.empty(tokens, ffn, device=device, dtype=torch.bfloat16) for _ in range(P)] for _ in range(layers)]
        self.dmid = [torch.empty(tokens, ffn, device=device, dtype=torch.bfloat16) for _ in range(P)]
        self.mean, self.rstd = [vector(tokens) for _ in range(layers + 1)], [vector(tokens) for _ in range(layers + 1)]
        self.dh, self.dy, self.dnext = rows(), rows(), rows()
        self.loss, self.lse = vector(tokens), vector(tokens)
        self.dtable = [torch.empty_like(t) for t in self.table]
        self.dgamma, self.dbeta = [vector(hidden) for _ in range(layers + 1)], [vector(hidden) for _ in range(layers + 1)]

    def forward(self, ids, targets):
        """Loss of every token (0 where the target is outside the vocabulary)."""
        api.compass_embedding(self.embed, ids, self.table, self.h[0])
        for i in range(self.layers + 1):
            # norm i also adds what MLP block i - 1 gave to the residual stream
            more = dict(residual=self.h[i - 1], summed=self.h[i]) if i else {}
            api.compass_layer_norm(self.norm, self.out[i - 1] if i else self.h[0], self.gamma[i], self.beta[i], self.y[i],
                                   mean=self.mean[i], rstd=self.rstd[i], **more)
            if i < self.layers:
                api.compass_mlp_block(self.mlp, self.y[i], self.w0[i], self.mid[i], self.w1[i], self.out[i], self.ws_mlp)
        api.compass_head_loss(self.head, self.y[-1], self.table, targets, self.loss, self.lse, self.ws_head)
        return self.loss

    def backward(self, ids, targets, dloss) -> None:
        """Gradients of the table, gammas and betas, from the gradient of every token's loss."""
        api.compass_head_loss_backward(self.head, self.y[-1], self.table, targets, self.lse, dloss, self.dy, self.dtable, self.ws_head_back)
        for i in range(self.layers, -1, -1):
            # self.dh: gradient of the residual stream behind norm i (none behind the last)
            api.compass_layer_norm_backward(self.norm, self.dy, self.h[i], self.gamma[i], self.mean[i], self.rstd[i], self.dnext,
                                            self.dgamma[i], self.dbeta[i], self.ws_norm, dsum=self.dh if i < self.layers else None)
            self.dh, self.dnext = self.dnext, self.dh
            if i:
                # through block i - 1: the same chain on the stored weights, the second one first
                api.compass_mlp_block(self.mlp_back, self.dh, self.w1[i - 1], self.dmid, self.w0[i - 1], self.dy, self.ws_mlp_back)
        api.compass_embedding_backward(self.embed, ids, self.dh, self.dtable, self.ws_embed)

    def parameters(self) -> List:
        return self.table + self.gamma + self.beta

    def gradients(self) -> List:
        return self.dtable + self.dgamma + self.dbeta

    def step(self, ids, targets, lr: float):
        """One step of plain gradient descent on the mean loss; returns that loss (on the device)."""
        valid = (targets >= 0) & (targets < self.V)
        dloss = valid.float() / valid.sum().clamp(min=1)
        mean = (self.forward(ids, targets) * dloss).sum()
        self.backward(ids, targets, dloss)
        for p, d in zip(self.parameters(), self.gradients()):
            p.add_(d, alpha=-lr)
        return mean

    def check(self) -> None:
        """Raises if a bounded device-side wait gave up (synchronises)."""
        for name, ws in (("head", self.ws_head), ("head backward", self.ws_head_back), ("mlp", self.ws_mlp), ("mlp backward", self.ws_mlp_back)):
            status, detail = api.compass_read_status(ws)
            if status != api.OK:
                raise api.CompassError(status, f"{name} (wait {detail})")


class TiedModel8:
    """The same model with root-mean-square norms and MLP blocks of 8-bit products, all of it trained."""

    def __init__(self, P: int, tokens: int, hidden: int, ffn: int, vocab: int, layers: int, seed: int = 0, device: str = "cuda"):
        import torch
        self.torch, self.P, self.M, self.H, self.F, self.V, self.layers = torch, P, tokens, hidden, ffn, vocab, layers
        g = torch.Generator(device=device).manual_seed(seed)
        normal = lambda scale, *shape: (torch.randn(*shape, generator=g, device=device) * scale).bfloat16()  # noqa: E731
        rows = lambda: [torch.empty(tokens // P, hidden, device=device, dtype=torch.bfloat16) for _ in range(P)]  # noqa: E731
        wide = lambda: [torch.empty(tokens, ffn, device=device, dtype=torch.bfloat16) for _ in range(P)]  # noqa: E731
        vector = lambda n: torch.empty(n, device=device)  # noqa: E731
        eight = lambda *a, **k: api.alloc_8bit(P, *a, device=device, **k)  # noqa: E731
        self.table = [normal(0.02, api.vocab_shard_rows(vocab, P, r), hidden) for r in range(P)]
        self.w0 = [[normal(hidden ** -0.5, ffn, hidden) for _ in range(P)] for _ in range(layers)]
        self.w1 = [[normal(0.5 * (P * ffn) ** -0.5, hidden, ffn) for _ in range(P)] for _ in range(layers)]
        self.gamma = [torch.ones(hidden, device=device) for _ in range(layers + 1)]

        self.embed = api.make_embedding(P, tokens, hidden, vocab, scale=hidden ** 0.5, accumulate=True)
        self.norm = api.make_rms_norm(P, tokens, hidden, param_dtype=api.DTYPE_FP32)
        self.head = api.make_head(P, tokens, hidden, vocab)
        gather, reduce = api.OP_AG_GEMM, api.OP_GEMM_RS
        self.up = api.make_problem(gather, P, tokens, ffn, hidden, dtype=api.DTYPE_E4M3)            # gather(y) * w0^T
        self.down = api.make_problem(reduce, P, tokens, hidden, ffn, dtype=api.DTYPE_E4M3)          # sum of mid * w1^T
        # gradients in E5M2, on the weights as they are stored
        self.down_back = api.make_problem(gather, P, tokens, ffn, hidden, dtype=api.DTYPE_E5M2, b_layout=api.B_KN)
        self.up_back = api.make_problem(reduce, P, tokens, hidden, ffn, dtype=api.DTYPE_E5M2, b_layout=api.B_KN)
        self.keep_w0 = api.make_quant(P, P * ffn, hidden, block_rows=128)
        self.keep_w1 = api.make_quant(P, P * hidden, ffn, block_rows=128)
        self.keep_mid = api.make_quant(P, P * tokens, ffn)
        self.keep_dmid = api.make_quant(P, P * tokens, ffn, format=api.DTYPE_E5M2)
        self.keep_dh = api.make_quant(P, tokens, hidden, format=api.DTYPE_E5M2)
        self.ws_embed = api.alloc_embedding_workspace(self.embed, device)
        self.ws_norm = api.alloc_rms_norm_workspace(self.norm, device)
        self.ws_head = api.alloc_head_workspace(self.head, device=device)
        self.ws_head_back = api.alloc_head_workspace(self.head, backward=True, device=device)
        self.ws = api.alloc_8bit_workspace(self.up, device)

        self.h = [rows() for _ in range(layers + 1)]                  # the residual stream, before each norm
        self.y8 = [eight(tokens // P, hidden) for _ in range(layers)] # after it
        self.y = rows()                                               # after the last
        self.out = [rows() for _ in range(layers)]                    # of the MLP blocks
        self.mid, self.mid8 = wide(), [eight(tokens, ffn) for _ in range(layers)]
        self.w0_8, self.w1_8 = [eight(ffn, hidden, block_rows=128) for _ in range(layers)], [eight(hidden, ffn, block_rows=128) for _ in range(layers)]
        self.dmid, self.dmid8 = wide(), eight(tokens, ffn, api.DTYPE_E5M2)
        self.dh8 = eight(tokens // P, hidden, api.DTYPE_E5M2)
        self.rstd = [vector(tokens) for _ in range(layers + 1)]
        self.dh, self.dy, self.dnext = rows(), rows(), rows()
        self.loss, self.lse = vector(tokens), vector(tokens)
        self.dtable = [torch.empty_like(t) for t in self.table]
        self.dgamma = [vector(hidden) for _ in range(layers + 1)]
        self.dw0, self.dw1 = [[[torch.empty_like(t) for t in w] for w in ws] for ws in (self.w0, self.w1)]

    def forward(self, ids, targets):
        """Loss of every token (0 where the target is outside the vocabulary)."""
        api.compass_embedding(self.embed, ids, self.table, self.h[0])
        for i in range(self.layers + 1):
            # norm i also adds what MLP block i - 1 gave to the residual stream
            x = self.out[i - 1] if i else self.h[0]
            more = dict(residual=self.h[i - 1], summed=self.h[i]) if i else {}
            if i == self.layers:
                api.compass_rms_norm(self.norm, x, self.gamma[i], Y=self.y, rstd=self.rstd[i], **more)
                break
            api.compass_rms_norm(self.norm, x, self.gamma[i], rstd=self.rstd[i], Y8=self.y8[i][0], scale=self.y8[i][1], **more)
            api.compass_quantize(self.keep_w0, self.w0[i], *self.w0_8[i])
            api.compass_quantize(self.keep_w1, self.w1[i], *self.w1_8[i])
            api.compass_ag_gemm_8bit(self.up, *self.y8[i], *self.w0_8[i], self.mid, self.ws)
            api.compass_quantize(self.keep_mid, self.mid, *self.mid8[i])
            api.compass_gemm_rs_8bit(self.down, *self.mid8[i], *self.w1_8[i], self.out[i], self.ws)
        api.compass_head_loss(self.head, self.y, self.table, targets, self.loss, self.lse, self.ws_head)
        return self.loss

    def backward(self, ids, targets, dloss) -> None:
        """Gradients of everything, from the gradient of every token's loss."""
        api.compass_head_loss_backward(self.head, self.y, self.table, targets, self.lse, dloss, self.dy, self.dtable, self.ws_head_back)
        for i in range(self.layers, -1, -1):
            # self.dh: gradient of the residual stream behind norm i (none behind the last)
            api.compass_rms_norm_backward(self.norm, self.dy, self.h[i], self.gamma[i], self.rstd[i], self.dnext, self.dgamma[i], self.ws_norm,
                                          dsum=self.dh if i < self.layers else None)
            self.dh, self.dnext = self.dnext, self.dh
            if i:
                k = i - 1
                api.compass_weight_grad_8bit(self.down, self.dh, *self.mid8[k], self.dw1[k], self.ws)
                api.compass_quantize(self.keep_dh, self.dh, *self.dh8)
                api.compass_ag_gemm_8bit(self.down_back, *self.dh8, *self.w1_8[k], self.dmid, self.ws)
                api.compass_weight_grad_8bit(self.up, self.dmid, *self.y8[k], self.dw0[k], self.ws)
                api.compass_quantize(self.keep_dmid, self.dmid, *self.dmid8)
                api.compass_gemm_rs_8bit(self.up_back, *self.dmid8, *self.w0_8[k], self.dy, self.ws)
        api.compass_embedding_backward(self.embed, ids, self.dh, self.dtable, self.ws_embed)

    def parameters(self) -> List:
        return self.table + self.gamma + [t for w in (self.w0, self.w1) for layer in w for t in layer]

    def gradients(self) -> List:
        return self.dtable + self.dgamma + [t for w in (self.dw0, self.dw1) for layer in w for t in layer]

    step = TiedModel.step

    def check(self) -> None:
        """Raises if a bounded device-side wait gave up (synchronises)."""
        for name, ws in (("head", self.ws_head), ("head backward", self.ws_head_back), ("8-bit products", self.ws)):
            status, detail = api.compass_read_status(ws)
            if status != api.OK:
                raise api.CompassError(status, f"{name} (wait {detail})")


def synthetic_batch(tokens: int, vocab: int, seed: int, device: str = "cuda"):
    """Token ids with frequencies like 1 / rank, each followed by a fixed successor; every tenth target is left out."""
    import torch
    g = torch.Generator(device=device).manual_seed(seed)
    u = torch.rand(tokens, generator=g, device=device, dtype=torch.float64)
    ids = ((vocab + 1.0) ** u).long().clamp_(1, vocab) - 1
    targets = (ids * 7 + 3) % vocab
    targets[::10] = -100
    return ids, targets


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("P", 4), ("tokens", 4096), ("hidden", 1024), ("ffn", 512), ("vocab", 32000), ("layers", 2), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--lr", type=float, default=0.2)
    ap.add_argument("--products", choices=("bf16", "8bit"), default="bf16")
    a = ap.parse_args()
    import torch
    model = (TiedModel8 if a.products == "8bit" else TiedModel)(a.P, a.tokens, a.hidden, a.ffn, a.vocab, a.layers)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for i in range(a.steps):
        ids, targets = synthetic_batch(a.tokens, a.vocab, i)
        begin.record()
        loss = model.step(ids, targets, a.lr)
        end.record()
        torch.cuda.synchronize()
        print(f"step {i}: loss {loss.item():.4f}, {begin.elapsed_time(end):.2f} ms")
    model.check()


if __name__ == "__main__":
    main()
