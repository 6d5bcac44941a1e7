"""The transformer's step on batches whose examples are mostly padding."""
import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild
from test_gpu_transformer import F64, Packed, batch, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


@pytest.mark.parametrize("dtype,bound", [(torch.bfloat16, 12 * 2.0 ** -8), (torch.float32, 5e-5)])  # as the whole batch's tests
@pytest.mark.parametrize("every", [2, 7])
def test_padded_batches(dev, every, dtype, bound):
    V, d, ff, nb, N, T = 64, 64, 128, 1, 49, 60
    m = Packed(V, d, ff, nb, N, T, heads=8, kv_heads=4, dtype=dtype, seed=5, cap=20.0, n_buckets=8, max_distance=20)
    m.table.normal_()
    tokens, targets, *m.packing = batch(V, N, T, dev, 2)
    empty = torch.arange(N, device=dev) % every != 0
    tokens[empty], targets[empty] = -1, -1
    P, per = reference(m, tokens, targets, *m.packing)
    m.gradients(tokens, targets)
    tda.tda_device_status()
    want = torch.autograd.grad(per.sum(), P)
    for g, x, p in zip(m.grads, want, m.params):
        assert float((g.to(F64) - x).norm()) <= bound * float(x.norm()) + 1e-9, tuple(p.shape)
    first = [g.clone() for g in m.grads]
    for _ in range(3):
        m.gradients(tokens, targets)
        tda.tda_device_status()
        assert all(torch.equal(a, b) for a, b in zip(first, m.grads))
