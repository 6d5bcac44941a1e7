"""The token model of capture.py: its whole step against torch's autograd in fp64 (fp32 model), the features of
its factors against the oracle, and the clipped update."""
import math

import numpy as np
import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild
from paper_2609_38767_gb300 import capture

pytestmark = pytest.mark.gpu
F64 = torch.float64


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


def batch(V, N, T, dev, seed=0):
    g = torch.Generator(device=dev).manual_seed(seed)
    seq = torch.randint(0, V, (N, T + 1), generator=g, device=dev)
    tokens, targets = seq[:, :T].int().contiguous(), seq[:, 1:].int().contiguous()
    tokens[1, T // 2:] = -1
    targets[1, T // 2:] = -1
    targets[2] = -1  # an example whose mask leaves nothing
    return tokens, targets


def reference(m, tokens, targets):
    """The same model in fp64 torch: loss and gradients by autograd, per example as well."""
    P = [p.detach().to(F64).requires_grad_(True) for p in m.params]
    t, y = tokens.reshape(-1).long(), targets.reshape(-1).long()
    h = P[0][t.clamp(min=0)] * (t >= 0).unsqueeze(1) * m.scale
    i = 1
    for _ in m.blocks:
        z = h @ P[i].t() + P[i + 1]
        h = h + torch.nn.functional.silu(z) @ P[i + 2].t() + P[i + 3]
        i += 4
    logp = torch.log_softmax(h @ P[i].t() + P[i + 1], 1)
    nll = -logp.gather(1, y.clamp(min=0).unsqueeze(1)).squeeze(1) * (y >= 0)
    n = (y.view(m.N, m.T) >= 0).sum(1).clamp(min=1)
    per = nll.view(m.N, m.T).sum(1) / n
    return P, per


@pytest.mark.parametrize("shape", [(96, 64, 128, 2, 6, 16), (200, 40, 72, 1, 5, 9)])
def test_step_against_autograd(dev, orc, shape):
    V, d, ff, nb, N, T = shape
    m = capture.TokenModel(V, d, ff, nb, N, T, dtype=torch.float32, max_norm=0.5, lr=0.25, seed=3)
    tokens, targets = batch(V, N, T, dev)
    P, per = reference(m, tokens, targets)
    loss = m.gradients(tokens, targets)
    tda.tda_device_status()
    total_loss = float(per.detach().sum())
    assert abs(float(loss) - total_loss) <= 1e-5 * total_loss
    want = torch.autograd.grad(per.sum(), P, retain_graph=True)
    for g, w in zip(m.grads, want):
        # fp32 products and sums of a few hundred terms through 2 nb + 1 layers
        assert float((g.to(F64) - w).norm()) <= 2e-5 * float(w.norm())
    # the factors that the step left, projected, are the projected per-example gradients
    k = 8
    phi = m.features(k, seed=7).cpu().numpy().astype(np.float64)
    for e in (0, 1, 2):
        rows = torch.autograd.grad(per[e], [P[1 + 2 * i] for i in range(len(m.linears))], retain_graph=True)
        for i, (x, gw) in enumerate(zip(m.linears, rows)):
            Sa = orc.proj_entries(7, i, 0, x.L.d_in, k).astype(np.float64)
            Sg = orc.proj_entries(7, i, 1, x.L.d_out, k).astype(np.float64)
            ref = (Sg.T @ gw.cpu().numpy() @ Sa / k).reshape(-1)
            got = phi[e, i * k * k:(i + 1) * k * k]
            assert np.linalg.norm(got - ref) <= 5e-5 * np.linalg.norm(ref) + 1e-12, (e, i)
    # clipped update
    before = [p.detach().to(F64).clone() for p in m.params]
    _, norm = m.step(tokens, targets)
    total = math.sqrt(sum(float((w ** 2).sum()) for w in want))
    assert abs(float(norm) - total) <= 2e-5 * total
    c = min(1.0, 0.5 / total)
    for p, b, w in zip(m.params, before, want):
        move = p.to(F64) - b
        assert float((move + 0.25 * c * w).norm()) <= 4e-5 * 0.25 * c * float(w.norm()) + 1e-7 * float(b.norm())


def test_bf16_model_learns_and_finds_twins(dev):
    torch.manual_seed(1)
    V, N, T = 256, 32, 24
    m = capture.TokenModel(V, 64, 128, 1, N, T, seed=5)
    pattern = torch.randint(0, V, (N // 2, 3), device=dev).repeat_interleave(2, 0)
    seq = pattern.repeat(1, T // 3 + 1)
    tokens, targets = seq[:, :T].int().contiguous(), seq[:, 1:T + 1].int().contiguous()
    losses = [float(m.step(tokens, targets)[0]) for _ in range(6)]
    tda.tda_device_status()
    assert all(b < a for a, b in zip(losses, losses[1:])), losses  # descent by small steps
    m.gradients(tokens, targets)
    phi = m.features(16)
    S = phi @ phi.t()
    S.fill_diagonal_(float("-inf"))
    assert bool((S.argmax(1) == (torch.arange(N, device=dev) ^ 1)).all())
