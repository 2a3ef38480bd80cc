"""Embedding, layer norm and output-layer loss launch on the current device: tensors of another one are refused by the binding
(stand-ins for tensors of two devices; nothing is launched and no GPU is needed)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api

BF16, F32, I64 = torch.bfloat16, torch.float32, torch.int64


class Tensor:
    """What the binding looks at."""
    is_cuda = True

    def __init__(self, dtype, *shape, device=0):
        self.dtype, self.shape, self.index, self.device = dtype, shape, device, f"cuda:{device}"

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def stride(self):
        return (1,) * len(self.shape)

    def numel(self):
        n = 1
        for k in self.shape:
            n *= k
        return n

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 0x10000


def rows(device):
    return [Tensor(BF16, 2, 16), Tensor(BF16, 2, 16, device=device)]


def table(device):
    return [Tensor(BF16, 5, 16), Tensor(BF16, 5, 16, device=device)]


ids, workspace = (lambda d: Tensor(I64, 4, device=d)), (lambda d: Tensor(torch.uint8, 1 << 20, device=d))
vector, param = (lambda d: Tensor(F32, 4, device=d)), (lambda d: Tensor(BF16, 16, device=d))
NORM, EMBED, HEAD = api.make_layer_norm(2, 4, 16), api.make_embedding(2, 4, 16, 10), api.make_head(2, 4, 16, 10)
CALLS = {
    "embedding": (lambda **t: api.compass_embedding(EMBED, **t), dict(ids=ids, W=table, Out=rows)),
    "embedding_backward": (lambda **t: api.compass_embedding_backward(EMBED, **t), dict(ids=ids, dOut=rows, dW=table, workspace=workspace)),
    "layer_norm": (lambda **t: api.compass_layer_norm(NORM, **t),
                   dict(X=rows, gamma=param, beta=param, Y=rows, mean=vector, rstd=vector, residual=rows, summed=rows)),
    "layer_norm_backward": (lambda **t: api.compass_layer_norm_backward(NORM, **t),
                            dict(dY=rows, X=rows, gamma=param, mean=vector, rstd=vector, dX=rows, dgamma=param, dbeta=param,
                                 workspace=workspace, dsum=rows)),
    "head_loss": (lambda **t: api.compass_head_loss(HEAD, **t),
                  dict(X=rows, W=table, targets=ids, loss=vector, lse=vector, workspace=workspace)),
    "head_loss_backward": (lambda **t: api.compass_head_loss_backward(HEAD, **t),
                           dict(X=rows, W=table, targets=ids, lse=vector, dloss=vector, dX=rows, dW=table, workspace=workspace)),
}


class Library:
    """Stands in for the loaded library and notes what reaches it."""

    def __init__(self):
        self.called = []

    def __getattr__(self, name):
        return lambda *a: self.called.append(name) or api.OK


@pytest.fixture
def library(monkeypatch):
    api.lib()
    fake = Library()
    monkeypatch.setattr(api, "lib", lambda: fake)
    monkeypatch.setattr(api, "_current_device", lambda: 0)
    monkeypatch.setattr(api, "_raw_stream", lambda device: 0)
    return fake


@pytest.mark.parametrize("call,name", [(c, n) for c, (_, names) in CALLS.items() for n in names])
def test_tensors_of_another_device_are_refused(library, call, name):
    run, names = CALLS[call]
    run(**{n: make(0) for n, make in names.items()})
    assert library.called == ["compass_" + call]
    with pytest.raises(ValueError, match="cuda:1"):
        run(**{n: make(int(n == name)) for n, make in names.items()})
    assert len(library.called) == 1


def test_workspaces_have_to_be_dense_and_on_the_gpu(library):
    run, names = CALLS["head_loss"]
    t = {n: make(0) for n, make in names.items()}
    for change in (dict(index=-1), dict(is_contiguous=lambda: False)):
        t["workspace"] = workspace(0)
        t["workspace"].__dict__.update(change)
        with pytest.raises(ValueError, match="workspace"):
            run(**t)
    assert library.called == []
