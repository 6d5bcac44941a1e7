"""The token model's host side (no GPU: the library's calls are replaced by fakes that record their arguments)."""
import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild
from paper_2609_38767_gb300 import capture


@pytest.fixture
def model(monkeypatch):
    tbuild.build()
    m = capture.TokenModel(50, 8, 16, 1, 3, 4, dtype=torch.float32, device="cpu")
    m.calls = []
    for name in ("tda_embedding_forward", "tda_embedding_backward", "tda_linear_forward", "tda_linear_backward",
                 "tda_grad_clip"):
        monkeypatch.setattr(tda, name, lambda *a, name=name: m.calls.append((name, a)))
    return m


def test_ids_are_read_as_what_they_are(model):
    for dtype, index in ((torch.int32, tda.TDA_I32), (torch.int64, tda.TDA_I64)):
        model.calls.clear()
        model.forward(torch.zeros((3, 4), dtype=dtype))
        model.backward(torch.zeros((12, 50)))
        name, a = model.calls[0]
        assert name == "tda_embedding_forward" and a[5] == index and a[6].dtype == dtype and a[7] == 12
        name, a = model.calls[-1]
        assert name == "tda_embedding_backward" and a[5] == index and a[6].dtype == dtype and a[7] == 12


def test_other_batches_are_refused(model):
    """A smaller batch would be read past its end, other types as if they were ids, host memory as the GPU's."""
    for tokens in (torch.zeros((2, 4), dtype=torch.int32), torch.zeros((3, 5), dtype=torch.int64),
                   torch.zeros((3, 4), dtype=torch.int16), torch.zeros((3, 4)),
                   torch.zeros((3, 4), dtype=torch.int32, device="meta")):
        with pytest.raises(ValueError):
            model.forward(tokens)
    assert not model.calls


def test_other_gradients_are_refused(model):
    model.forward(torch.zeros((3, 4), dtype=torch.int32))
    model.calls.clear()
    for g in (torch.zeros((11, 50)), torch.zeros((12, 49)), torch.zeros((12, 50), dtype=torch.bfloat16),
              torch.zeros((50, 12)).t(), torch.zeros((12, 50), device="meta")):
        with pytest.raises(ValueError):
            model.backward(g)
    assert not model.calls
