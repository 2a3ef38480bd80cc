"""Embedding, layer norm and output-layer loss: what the C ABI and the binding refuse, and their workspaces (no GPU)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api

BAD = [
    (dict(P=0), api.ERR_INVALID_ARG),
    (dict(P=17), api.ERR_UNSUPPORTED),
    (dict(M=-1), api.ERR_SHAPE),
    (dict(P=4, M=6), api.ERR_SHAPE),
    (dict(hidden=0), api.ERR_SHAPE),
    (dict(M=2 ** 31, P=1), api.ERR_UNSUPPORTED),
    (dict(dtype=7), api.ERR_UNSUPPORTED),
]
VOCAB = [(dict(vocab=0), api.ERR_SHAPE), (dict(vocab=2 ** 31), api.ERR_UNSUPPORTED), (dict(index_dtype=2), api.ERR_INVALID_ARG),
         (dict(grad_dtype=3), api.ERR_UNSUPPORTED)]
DESCRIBED = {
    "embedding": (api.make_embedding, dict(P=2, M=4, hidden=16, vocab=10), BAD + VOCAB),
    "layer_norm": (api.make_layer_norm, dict(P=2, M=4, hidden=16),
                   BAD + [(dict(param_dtype=5), api.ERR_UNSUPPORTED), (dict(eps=-1.0), api.ERR_INVALID_ARG),
                          (dict(eps=float("nan")), api.ERR_INVALID_ARG)]),
    "head": (api.make_head, dict(P=2, M=4, hidden=16, vocab=10),
             BAD + VOCAB + [(dict(dtype=api.DTYPE_FP32), api.ERR_UNSUPPORTED), (dict(hidden=12), api.ERR_ALIGNMENT),
                            (dict(label_smoothing=1.0), api.ERR_INVALID_ARG), (dict(label_smoothing=-0.1), api.ERR_INVALID_ARG),
                            (dict(label_smoothing=float("nan")), api.ERR_INVALID_ARG), (dict(logit_scale=float("inf")), api.ERR_INVALID_ARG),
                            (dict(logit_scale=float("nan")), api.ERR_INVALID_ARG)]),
}
SIZES = {"embedding": api.compass_embedding_workspace_bytes, "layer_norm": api.compass_layer_norm_workspace_bytes,
         "head": api.compass_head_workspace_bytes}


@pytest.mark.parametrize("name,change,status", [(n, c, s) for n, (_, _, bad) in DESCRIBED.items() for c, s in bad])
def test_descriptions_that_are_refused(name, change, status):
    make, good, _ = DESCRIBED[name]
    SIZES[name](make(**good))
    with pytest.raises(api.CompassError) as e:
        SIZES[name](make(**{**good, **change}))
    assert e.value.status == status


def test_null_descriptions():
    n = C.c_size_t()
    L = api.lib()
    assert L.compass_embedding_workspace_bytes(None, C.byref(n)) == api.ERR_INVALID_ARG
    assert L.compass_layer_norm_workspace_bytes(None, C.byref(n)) == api.ERR_INVALID_ARG
    assert L.compass_head_workspace_bytes(None, 0, C.byref(n)) == api.ERR_INVALID_ARG
    assert L.compass_head_workspace_bytes(C.byref(api.make_head(1, 1, 8, 1)), 0, None) == api.ERR_INVALID_ARG


def test_struct_layouts_match_the_header():
    assert C.sizeof(api.Embed) == 4 * 4 + 3 * 8 + 2 * 4 and api.Embed.M.offset == 16 and api.Embed.accumulate.offset == 44
    assert C.sizeof(api.Norm) == 4 * 4 + 2 * 8 and api.Norm.eps.offset == 12
    assert C.sizeof(api.Head) == 4 * 4 + 3 * 8 + 2 * 4 and api.Head.label_smoothing.offset == 44


# Addresses that are never read: every call below is refused on the host.  ODD: on no element's boundary; HALF: not on 16 bytes.
A, ODD, HALF = 0x10000, 0x10001, 0x10008


def ptrs(*p):
    return (C.c_void_p * len(p))(*p)


def test_embedding_calls_that_are_refused():
    e, L = api.make_embedding(2, 4, 16, 10), api.lib()
    good, null, odd = ptrs(A, A), ptrs(A, None), ptrs(A, ODD)
    need = api.compass_embedding_workspace_bytes(e)
    forward = lambda ids=A, w=good, out=good: L.compass_embedding(C.byref(e), ids, w, out, None)  # noqa: E731
    back = lambda ids=A, d=good, w=good, ws=A, n=need: L.compass_embedding_backward(C.byref(e), ids, d, w, ws, n, None)  # noqa: E731
    assert forward(ids=None) == forward(w=None) == forward(out=None) == forward(w=null) == forward(out=null) == api.ERR_INVALID_ARG
    assert forward(ids=A + 4) == forward(w=odd) == forward(out=odd) == api.ERR_ALIGNMENT
    assert back(ids=None) == back(d=None) == back(w=null) == back(ws=None) == api.ERR_INVALID_ARG
    assert back(d=odd) == back(w=odd) == back(ws=A + 128) == api.ERR_ALIGNMENT
    assert back(n=need - 1) == api.ERR_BUFFER_TOO_SMALL
    # a shard without rows may be NULL, but not one with rows: 10 rows over 4 ranks are 3, 3, 3, 1; 5 are 2, 2, 1, 0
    e5 = api.make_embedding(4, 4, 16, 5)
    four = ptrs(A, A, A, A)
    assert L.compass_embedding(C.byref(e5), A, ptrs(A, A, None, None), four, None) == api.ERR_INVALID_ARG
    assert L.compass_embedding(C.byref(e5), A + 1, ptrs(A, A, A, None), four, None) == api.ERR_ALIGNMENT


def test_layer_norm_calls_that_are_refused():
    n, L = api.make_layer_norm(2, 4, 16), api.lib()
    good, null, odd = ptrs(A, A), ptrs(None, A), ptrs(A, ODD)
    need = api.compass_layer_norm_workspace_bytes(n)

    def forward(x=good, r=None, g=A, b=A, s=None, y=good, mean=None, rstd=None):
        return L.compass_layer_norm(C.byref(n), x, r, g, b, s, y, mean, rstd, None)

    def back(dy=good, x=good, g=A, mean=A, rstd=A, ds=None, dx=good, dg=A, db=A, ws=A, size=need):
        return L.compass_layer_norm_backward(C.byref(n), dy, x, g, mean, rstd, ds, dx, dg, db, ws, size, None)

    assert forward(x=None) == forward(x=null) == forward(y=None) == forward(r=good) == forward(s=good) == api.ERR_INVALID_ARG
    assert forward(x=odd) == forward(r=odd, s=good) == forward(g=ODD) == forward(b=ODD) == forward(mean=A + 2) == api.ERR_ALIGNMENT
    assert back(dy=None) == back(x=null) == back(dx=None) == back(mean=None) == back(rstd=None) == back(ws=None) == api.ERR_INVALID_ARG
    assert back(ds=null) == api.ERR_INVALID_ARG
    assert back(ds=odd) == back(dg=ODD) == back(db=ODD) == back(ws=ODD) == api.ERR_ALIGNMENT
    assert back(size=need - 1) == api.ERR_BUFFER_TOO_SMALL


def test_head_calls_that_are_refused():
    h, L = api.make_head(2, 4, 16, 10), api.lib()
    good, null, odd = ptrs(A, A), ptrs(None, A), ptrs(A, HALF)
    need, need_back = api.compass_head_workspace_bytes(h), api.compass_head_workspace_bytes(h, True)

    def forward(x=good, w=good, y=A, loss=A, lse=A, ws=A, n=need):
        return L.compass_head_loss(C.byref(h), x, w, y, loss, lse, ws, n, None)

    def back(x=good, w=good, y=A, lse=A, dl=A, dx=good, dw=good, ws=A, n=need_back):
        return L.compass_head_loss_backward(C.byref(h), x, w, y, lse, dl, dx, dw, ws, n, None)

    for call in (forward, back):
        assert call(x=None) == call(x=null) == call(w=None) == call(w=null) == call(y=None) == call(ws=None) == api.ERR_INVALID_ARG
        assert call(x=odd) == call(w=odd) == call(y=A + 4) == call(ws=A + 64) == api.ERR_ALIGNMENT
        assert call(n=need - 1) == api.ERR_BUFFER_TOO_SMALL
        assert call(lse=None) == api.ERR_INVALID_ARG and call(lse=A + 2) == api.ERR_ALIGNMENT
    assert forward(loss=None) == back(dl=None) == back(dx=None) == back(dw=null) == api.ERR_INVALID_ARG
    assert back(dx=odd) == back(dw=odd) == api.ERR_ALIGNMENT


def test_workspaces_are_bounded():
    """The gradient of the logits takes 256 MB at a time, whatever the vocabulary, not tokens * vocabulary."""
    big = api.compass_head_workspace_bytes(api.make_head(8, 8192, 4096, 128000), True)
    rows, sums = 8192 * 4096 * 2, 8192 * 4096 * 4
    assert big < rows + sums + (256 << 20) + (1 << 20)
    assert api.compass_head_workspace_bytes(api.make_head(8, 8192, 4096, 1024000), True) < big + (1 << 20)
    assert api.compass_head_workspace_bytes(api.make_head(1, 0, 64, 100), True) < 1 << 20
    # forward: 16 bytes per row and 256 vocabulary columns beside the gathered rows (24 with label smoothing)
    forward = api.compass_head_workspace_bytes(api.make_head(8, 8192, 4096, 128000))
    assert forward < rows + 8192 * 504 * 16 + (1 << 20)


def test_the_binding_refuses_tensors():
    """Type, shape, layout and device are looked at before the library is called."""
    n, e, h = api.make_layer_norm(2, 4, 16), api.make_embedding(2, 4, 16, 10), api.make_head(2, 4, 16, 10)
    x = [torch.zeros(2, 16, dtype=torch.bfloat16) for _ in range(2)]
    w = [torch.zeros(5, 16, dtype=torch.bfloat16) for _ in range(2)]
    ids, v = torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    ws = torch.zeros(1024, dtype=torch.uint8)
    for call in (lambda: api.compass_layer_norm(n, x, None, None, x),                                          # on the CPU
                 lambda: api.compass_layer_norm(n, x[:1], None, None, x),                                      # one shard of two
                 lambda: api.compass_layer_norm(n, [t.float() for t in x], None, None, x),
                 lambda: api.compass_embedding(e, ids, w, x),
                 lambda: api.compass_embedding(e, ids.int(), w, x),
                 lambda: api.compass_embedding_backward(e, ids, x, w[:1], ws),
                 lambda: api.compass_head_loss(h, x, w, ids, v, v, ws),
                 lambda: api.compass_head_loss_backward(h, x, w, ids, v, v, x, w, ws)):
        with pytest.raises(ValueError):
            call()
    for kind in (5, -1):
        with pytest.raises(ValueError):
            api._torch_dtype(kind)


def test_vocabulary_shards():
    for vocab, P in ((10, 4), (5, 4), (1, 16), (128000, 8), (32001, 16)):
        rows = [api.vocab_shard_rows(vocab, P, r) for r in range(P)]
        assert sum(rows) == vocab and rows == sorted(rows, reverse=True) and rows[0] == -(-vocab // P)
