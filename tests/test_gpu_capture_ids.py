"""The token model of capture.py on ids of either width."""
import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild
from paper_2609_38767_gb300 import capture

pytestmark = pytest.mark.gpu


def test_ids_of_64_bits():
    """torch's default ids give what the same ids in 32 bits give, bit for bit; padding and an empty example among them."""
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    V, N, T = 96, 6, 16
    g = torch.Generator(device="cuda").manual_seed(0)
    seq = torch.randint(0, V, (N, T + 1), generator=g, device="cuda")
    tokens, targets = seq[:, :T].contiguous(), seq[:, 1:].contiguous()
    tokens[1, T // 2:], targets[1, T // 2:], targets[2] = -1, -1, -1
    got = []
    for dtype in (torch.int32, torch.int64):
        m = capture.TokenModel(V, 64, 128, 1, N, T, dtype=torch.float32, seed=3)
        loss = m.gradients(tokens.to(dtype), targets)
        got.append([loss.clone()] + [x.clone() for x in m.grads])
    tda.tda_device_status()
    assert all(bool(torch.isfinite(a).all()) and torch.equal(a, b) for a, b in zip(*got))
