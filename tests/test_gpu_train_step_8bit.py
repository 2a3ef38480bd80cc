"""The tied-embedding model with 8-bit products: every operator of a step against 64 bits on what it was given, and the whole
gradients against the chain rule in 64 bits."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api
from paper_2609_10549_b200.train_step import TiedModel8, synthetic_batch
from tests.eight_bit import kept, values

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8      # half a step of BF16
CASES = [(1, 64, 64, 32, 100, 1), (4, 512, 256, 144, 1001, 1), (2, 700, 272, 528, 333, 1), (8, 2048, 512, 64, 700, 1)]


def step(P, tokens, hidden, ffn, vocab, layers):
    model = TiedModel8(P, tokens, hidden, ffn, vocab, layers, seed=3)
    ids, targets = synthetic_batch(tokens, vocab, 1)
    ids[5 % tokens] = -1
    dloss = torch.rand(tokens, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) / tokens
    loss = model.forward(ids, targets).clone()
    model.backward(ids, targets, dloss)
    model.check()
    return model, ids, targets, dloss, loss


def near_product(got, a, b, terms, add=None, half=HALF):
    """got = a @ b (+ add), one rounding and one unit of FP32 for every product that is added."""
    want, size = a @ b, a.abs() @ b.abs()
    if add is not None:
        want, size = want + add, size + add.abs()
    assert ((got.double() - want).abs() <= half * want.abs() + terms * 2.0 ** -23 * size).all()


@pytest.mark.parametrize("P,tokens,hidden,ffn,vocab,layers", CASES)
def test_every_operator_on_what_it_was_given(P, tokens, hidden, ffn, vocab, layers):
    m, ids, targets, dloss, loss = step(P, tokens, hidden, ffn, vocab, layers)
    cat = lambda t: torch.cat(list(t))  # noqa: E731
    eight = lambda pair, b=1: [values(q, s, b) for q, s in zip(*pair)]  # noqa: E731
    # the norm's output in 8 bits is that of the FP32 norm, but where the last bit tips it over
    h = cat(m.h[0]).double()
    y = h * (h.square().mean(1, keepdim=True) + m.norm.eps).rsqrt() * m.gamma[0].double()
    assert (cat(eight(m.y8[0])) == kept(y, api.DTYPE_E4M3)[1]).double().mean() > 0.999
    # weights and activations in 8 bits: the very bits
    for full, pair, b, f in ((m.w0[0], m.w0_8[0], 128, api.DTYPE_E4M3), (m.w1[0], m.w1_8[0], 128, api.DTYPE_E4M3), (m.mid, m.mid8[0], 1, api.DTYPE_E4M3),
                             (m.dmid, m.dmid8, 1, api.DTYPE_E5M2), (m.dnext, m.dh8, 1, api.DTYPE_E5M2)):
        for t, v in zip(full, eight(pair, b)):
            assert torch.equal(v, kept(t, f, b)[1])
    y8, w0, w1 = cat(eight(m.y8[0])), eight(m.w0_8[0], 128), eight(m.w1_8[0], 128)
    mid8, dh8, dmid8 = eight(m.mid8[0]), cat(eight(m.dh8)), eight(m.dmid8)
    dh = cat(m.dnext)      # the gradient behind the block (the last norm's backward swapped it there)
    for r in range(P):
        near_product(m.mid[r], y8, w0[r].T, hidden)
        near_product(m.dmid[r], dh8, w1[r], hidden)
        near_product(m.dw0[0][r], m.dmid[r].double().T, y8, tokens)
        near_product(m.dw1[0][r], dh.double().T, mid8[r], tokens)
    near_product(cat(m.out[0]), torch.cat(mid8, 1), torch.cat([w.T for w in w1]), P * ffn)
    near_product(cat(m.dy), torch.cat(dmid8, 1), torch.cat(w0), P * ffn)
    assert torch.equal(cat(m.h[1]), (cat(m.out[0]).float() + cat(m.h[0]).float()).bfloat16())


@pytest.mark.parametrize("P,tokens,hidden,ffn,vocab,layers", CASES + [(2, 256, 128, 64, 200, 3)])
def test_gradients(P, tokens, hidden, ffn, vocab, layers):
    """The chain rule in 64 bits with the same tensors kept in 8 bits.  Beside the roundings to BF16, of which about six a layer and
    direction lie between a gradient and the loss (2^-9 on average, twice over for what the norms make of them), a difference of 2^-9
    tips an element of a tensor kept in 8 bits over with a chance of 2^-6 (E4M3's steps are 2^-3), by such a step at most, 0.6 of it
    on average: 2^-3 * 2^-3 * 0.6 = 0.0094, and 0.0133 for E5M2; two of each a layer: 0.023, and twice that."""
    m, ids, targets, dloss, loss = step(P, tokens, hidden, ffn, vocab, layers)
    D = torch.float64
    table = torch.cat(m.table).double()
    gamma = [g.double() for g in m.gamma]
    w0 = [[kept(w, api.DTYPE_E4M3, 128)[1] for w in layer] for layer in m.w0]
    w1 = [[kept(w, api.DTYPE_E4M3, 128)[1] for w in layer] for layer in m.w1]
    h = [table[ids.clamp(min=0)] * m.embed.scale * (ids >= 0)[:, None]]
    y8, mid8 = [], []
    norm = lambda x, g: x * (x.square().mean(1, keepdim=True) + m.norm.eps).rsqrt() * g  # noqa: E731
    for i in range(layers):
        y8.append(kept(norm(h[i], gamma[i]), api.DTYPE_E4M3)[1])
        mid8.append([kept(y8[i] @ w.T, api.DTYPE_E4M3)[1] for w in w0[i]])
        h.append(h[i] + sum(a @ w.T for a, w in zip(mid8[i], w1[i])))
    y = norm(h[-1], gamma[-1])
    z = y @ table.T
    want_loss = torch.nn.functional.cross_entropy(z, targets, ignore_index=-100, reduction="none")
    valid = targets >= 0
    dz = torch.softmax(z, 1)
    dz[valid, targets[valid]] -= 1
    dz *= (dloss.double() * valid)[:, None]
    dtable, dy, dh = dz.T @ y, dz @ table, torch.zeros_like(y)
    dgamma, dw0, dw1 = [None] * (layers + 1), [None] * layers, [None] * layers

    def norm_back(dy, x, g):
        r = (x.square().mean(1, keepdim=True) + m.norm.eps).rsqrt()
        xh, v = x * r, dy * g
        return r * (v - xh * (v * xh).mean(1, keepdim=True)), (dy * xh).sum(0)

    for i in range(layers, -1, -1):
        dx, dgamma[i] = norm_back(dy, h[i], gamma[i])
        dh = dh + dx
        if i:
            k = i - 1
            dw1[k] = [dh.T @ a for a in mid8[k]]
            dh8 = kept(dh, api.DTYPE_E5M2)[1]
            dmid = [dh8 @ w for w in w1[k]]
            dw0[k] = [d.T @ y8[k] for d in dmid]
            dy = sum(kept(d, api.DTYPE_E5M2)[1] @ w for d, w in zip(dmid, w0[k]))
    back = torch.zeros_like(table)
    back.index_add_(0, ids[ids >= 0], dh[ids >= 0] * m.embed.scale)
    dtable += back
    bound = ((4 * 2.0 ** -9) ** 2 * 12 * (layers + 1) + layers * (2 * 0.023) ** 2) ** 0.5
    assert (loss.to(D) - want_loss).norm() <= bound * want_loss.norm()
    got = [torch.cat(m.dtable)] + m.dgamma + [t for w in (m.dw0, m.dw1) for layer in w for t in layer]
    want = [dtable] + dgamma + [t for w in (dw0, dw1) for layer in w for t in layer]
    for a, b in zip(got, want):
        assert (a.to(D) - b).norm() <= bound * b.norm()


def test_steps_run_and_replay():
    """Steps in a row, and the same step captured and replayed: the same bits."""
    model, other = (TiedModel8(2, 512, 128, 64, 300, 2, seed=1) for _ in range(2))
    ids, targets = synthetic_batch(512, 300, 2)
    before = api.kernel_launch_count()
    for _ in range(2):
        loss = model.step(ids, targets, 0.1)
    assert api.kernel_launch_count() - before >= 2 * 2 * 12
    model.check()
    assert torch.isfinite(loss)
    other.step(ids, targets, 0.1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = other.step(ids, targets, 0.1)
    graph.replay()
    torch.cuda.synchronize()
    other.check()
    assert torch.equal(loss, replayed)
    for a, b in zip(model.parameters(), other.parameters()):
        assert torch.equal(a, b)
