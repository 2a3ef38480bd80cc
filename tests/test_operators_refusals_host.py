"""Descriptions that no library would take give the binding's errors in calls too, not a KeyError or a division by zero."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10549_b200 import api


@pytest.fixture
def here(monkeypatch):
    api.lib()
    monkeypatch.setattr(api, "_current_device", lambda: -1)       # the device of CPU tensors
    monkeypatch.setattr(api, "_raw_stream", lambda device: 0)


def tensors():
    x = [torch.zeros(4, 16, dtype=torch.bfloat16)]
    w = [torch.zeros(10, 16, dtype=torch.bfloat16)]
    return x, w, torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(1 << 20, dtype=torch.uint8)


def test_unknown_types_of_ids_and_targets(here):
    x, w, ids, v, ws = tensors()
    e, h = api.make_embedding(1, 4, 16, 10, index_dtype=2), api.make_head(1, 4, 16, 10, index_dtype=-1)
    for call in (lambda: api.compass_embedding(e, ids, w, x), lambda: api.compass_embedding_backward(e, ids, x, w, ws),
                 lambda: api.compass_head_loss(h, x, w, ids, v, v, ws),
                 lambda: api.compass_head_loss_backward(h, x, w, ids, v, v, x, w, ws)):
        with pytest.raises(ValueError, match="index type"):
            call()


def test_no_ranks(here):
    _, _, ids, v, ws = tensors()
    e, n, h = api.make_embedding(0, 4, 16, 10), api.make_layer_norm(0, 4, 16), api.make_head(0, 4, 16, 10)
    for call in (lambda: api.compass_embedding(e, ids, [], []), lambda: api.compass_layer_norm(n, [], None, None, []),
                 lambda: api.compass_head_loss(h, [], [], ids, v, v, ws)):
        with pytest.raises(api.CompassError) as err:
            call()
        assert err.value.status == api.ERR_INVALID_ARG
