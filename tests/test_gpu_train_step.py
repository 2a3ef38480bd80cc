"""The tied-embedding model: its gradients against automatic differentiation in 64 bits, and a few steps that learn."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from paper_2609_10549_b200.train_step import TiedModel, synthetic_batch

pytestmark = pytest.mark.gpu


def reference(model, ids, targets, dloss):
    """Loss per token and gradients by torch in 64 bits, from the model's weights."""
    table = torch.cat(model.table).double().requires_grad_()
    gamma = [g.double().requires_grad_() for g in model.gamma]
    beta = [b.double().requires_grad_() for b in model.beta]
    h = table[ids.clamp(min=0)] * model.embed.scale * (ids >= 0)[:, None]
    for i in range(model.layers + 1):
        y = torch.nn.functional.layer_norm(h, (model.H,), gamma[i], beta[i], 1e-5)
        if i < model.layers:
            for w0, w1 in zip(model.w0[i], model.w1[i]):
                h = h + (y @ w0.double().T) @ w1.double().T
    loss = torch.nn.functional.cross_entropy(y @ table.T, targets, ignore_index=-100, reduction="none")
    (loss * dloss.double()).sum().backward()
    return loss.detach(), [table.grad] + [g.grad for g in gamma] + [b.grad for b in beta]


@pytest.mark.parametrize("P,tokens,hidden,ffn,vocab,layers", [(1, 64, 64, 32, 100, 1), (4, 512, 256, 128, 1001, 2), (2, 4, 8, 8, 3, 3)])
def test_gradients(P, tokens, hidden, ffn, vocab, layers):
    """Every stored tensor between two operators is rounded to BF16 (2^-8 relative at most, 2^-9 on average): about six of them
    a layer and direction lie between a gradient and the loss, whose errors add up like their squares, and twice that covers
    what the norms make of them: relative error of a whole gradient within 2 * 2^-9 * sqrt(6 * (layers + 1) * 2) * 2."""
    model = TiedModel(P, tokens, hidden, ffn, vocab, layers, seed=3)
    ids, targets = synthetic_batch(tokens, vocab, 1)
    ids[5 % tokens] = -1
    dloss = torch.rand(tokens, device="cuda") / tokens
    loss = model.forward(ids, targets).clone()
    model.backward(ids, targets, dloss)
    model.check()
    want_loss, want = reference(model, ids, targets, dloss)
    bound = 4 * 2.0 ** -9 * (12 * (layers + 1)) ** 0.5
    assert (loss.double() - want_loss).norm() <= bound * want_loss.norm()
    for got, exact in zip([torch.cat(model.dtable)] + model.dgamma + model.dbeta, want):
        assert (got.double() - exact).norm() <= bound * exact.norm()


def test_steps_learn():
    model = TiedModel(2, 1024, 128, 64, 500, 1, seed=1)
    ids, targets = synthetic_batch(1024, 500, 2)
    before = api.kernel_launch_count()
    losses = [model.step(ids, targets, 0.3).item() for _ in range(30)]
    model.check()
    assert api.kernel_launch_count() - before >= 30 * 12
    assert losses[0] > 5.5 and losses[-1] < 0.6 * losses[0], losses
