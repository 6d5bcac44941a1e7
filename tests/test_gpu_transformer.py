"""The transformer of capture.py, where attention, ranges, norms, linears, embedding and clipping run together as a program
uses them: its gradients against autograd in fp64, the features of its factors, its update, and the command."""
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
    documents = (torch.rand((N, T), generator=g, device=dev) < 0.15).int().cumsum(1).int().contiguous()
    prefix = (torch.rand((N, T), generator=g, device=dev) < 0.6).int().contiguous()
    return tokens, targets, documents, prefix


def reference(m, tokens, targets, documents, prefix):
    """The same model in fp64 torch, the masks by loops over the tokens."""
    P = [p.detach().to(F64).requires_grad_(True) for p in m.params]
    at = {id(p): q for p, q in zip(m.params, P)}
    w = lambda x: at[id(x)]  # noqa: E731
    N, T, L = m.N, m.T, m.L
    t, y = tokens.reshape(-1).long(), targets.reshape(-1).long()
    seen = torch.zeros((N, T, T), dtype=torch.bool)
    tok, doc, pre = tokens.cpu(), documents.cpu(), prefix.cpu()
    for n in range(N):
        ids = [int(doc[n, i]) if tok[n, i] >= 0 else -1 for i in range(T)]
        for i in range(T):
            if ids[i] < 0:
                continue
            s = i
            while s and ids[s - 1] == ids[i]:
                s -= 1
            p = s
            while p < T and ids[p] == ids[i] and pre[n, p]:
                p += 1
            seen[n, i, s:max(i + 1, p)] = True
    seen = seen.to(m.E.device)
    norm = lambda x, g: x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-5) * g  # noqa: E731
    H, KV, hd = L.heads, L.kv_heads, L.head_dim
    apart = torch.arange(T, device=m.E.device)[:, None] - torch.arange(T, device=m.E.device)[None]
    R = L.max_distance
    h = w(m.E)[t.clamp(min=0)] * (t >= 0).unsqueeze(1) * m.scale
    for (qkv, out), (n1, n2), (up, down) in zip(m.around, m.norms, m.blocks):
        x = (norm(h, w(n1.w)) @ w(qkv.W).t() + w(qkv.b)).view(N, T, H + 2 * KV, hd).transpose(1, 2)
        q, k, v = x[:, :H], x[:, H:H + KV].repeat_interleave(H // KV, 1), x[:, H + KV:].repeat_interleave(H // KV, 1)
        s = q @ k.transpose(2, 3) * hd ** -0.5
        if L.cap:
            s = L.cap * torch.tanh(s / L.cap)
        if m.table is not None:
            s = s + w(m.table)[m.bucket.long()[apart.clamp(-R, R) + R]].permute(2, 0, 1)
        s = torch.where(seen[:, None], s, -math.inf)
        p = torch.softmax(torch.where(seen.any(2)[:, None, :, None], s, 0.0), 3) * seen[:, None]
        h = h + (p @ v).transpose(1, 2).reshape(N * T, H * hd) @ w(out.W).t() + w(out.b)
        u = torch.nn.functional.silu(norm(h, w(n2.w)) @ w(up.W).t() + w(up.b))
        h = h + u @ w(down.W).t() + w(down.b)
    logp = torch.log_softmax(norm(h, w(m.last.w)) @ w(m.head.W).t() + w(m.head.b), 1)
    nll = -logp.gather(1, y.clamp(min=0).unsqueeze(1)).squeeze(1) * (y >= 0)
    per = nll.view(N, T).sum(1) / (y.view(N, T) >= 0).sum(1).clamp(min=1)
    return P, per


class Packed(capture.TransformerModel):
    """The step's calls with documents and prefixes."""

    def forward(self, tokens, documents=None, prefix=None):
        return super().forward(tokens, *self.packing)


def check_features(orc, m, P, per, k=8):
    phi = m.features(k, seed=7).cpu().numpy().astype(np.float64)
    for e in (0, 1, 2):
        rows = torch.autograd.grad(per[e], [P[1 + 2 * i] for i in range(len(m.linears))], retain_graph=True, allow_unused=True)
        for i, (x, gw) in enumerate(zip(m.linears, rows)):
            Sa = orc.proj_entries(7, i, 0, x.L.d_in, k).astype(np.float64)
            Sg = orc.proj_entries(7, i, 1, x.L.d_out, k).astype(np.float64)
            ref = (Sg.T @ gw.cpu().numpy() @ Sa / k).reshape(-1)
            got = phi[e, i * k * k:(i + 1) * k * k]
            assert np.linalg.norm(got - ref) <= 1e-4 * np.linalg.norm(ref) + 1e-9, (e, i)


@pytest.mark.parametrize("shape,more", [((96, 64, 128, 2, 6, 16), dict(heads=4, kv_heads=2, cap=2.0)),
                                        ((50, 40, 72, 1, 4, 70), dict(heads=5, n_buckets=0)),
                                        ((64, 32, 64, 2, 3, 33), dict(heads=2, head_dim=24, n_buckets=7, max_distance=9))])
def test_step_against_autograd(dev, orc, shape, more):
    V, d, ff, nb, N, T = shape
    m = Packed(V, d, ff, nb, N, T, dtype=torch.float32, max_norm=0.5, lr=0.25, seed=3, **more)
    for pair in m.norms:
        for x in pair:
            x.w.uniform_(0.5, 1.5)
    if m.table is not None:
        m.table.normal_()
    tokens, targets, *m.packing = batch(V, N, T, dev)
    P, per = reference(m, tokens, targets, *m.packing)
    loss = m.gradients(tokens, targets)
    tda.tda_device_status()
    total = float(per.detach().sum())
    assert abs(float(loss) - total) <= 1e-5 * total
    want = torch.autograd.grad(per.sum(), P, retain_graph=True)
    for g, x in zip(m.grads, want):
        # fp32 products and sums of a few hundred terms, 2^-24 each, through some ten layers
        assert float((g.to(F64) - x).norm()) <= 5e-5 * float(x.norm()) + 1e-9
    if V % 4 == 0:  # the projection takes widths in fours
        check_features(orc, m, P, per)
    before = [p.detach().to(F64).clone() for p in m.params]
    _, norm = m.step(tokens, targets)
    total = math.sqrt(sum(float((x ** 2).sum()) for x in want))
    assert abs(float(norm) - total) <= 5e-5 * total
    c = min(1.0, 0.5 / total)
    for p, b, x in zip(m.params, before, want):
        move = p.to(F64) - b
        assert float((move + 0.25 * c * x).norm()) <= 1e-4 * 0.25 * c * float(x.norm()) + 1e-7 * float(b.norm()) + 1e-9


def test_bf16_step_against_autograd(dev):
    """The tensor-core kernels in a row: every gradient is near the fp64 model's of the same weights. Each layer rounds its
    outputs and its gradients to bf16 (2^-9 on average), about a dozen times on the way to any weight."""
    V, d, ff, nb, N, T = 128, 128, 256, 1, 4, 200
    m = Packed(V, d, ff, nb, N, T, heads=4, kv_heads=2, seed=5, cap=20.0)
    m.table.normal_()
    tokens, targets, *m.packing = batch(V, N, T, dev, 2)
    P, per = reference(m, tokens, targets, *m.packing)
    m.gradients(tokens, targets)
    tda.tda_device_status()
    want = torch.autograd.grad(per.sum(), P)
    for g, x, p in zip(m.grads, want, m.params):
        assert float((g.to(F64) - x).norm()) <= 12 * 2.0 ** -8 * float(x.norm()) + 1e-9, tuple(p.shape)


def test_captured_step(dev):
    """Forward and backward pass captured into a graph and replayed on new tokens give what the calls give."""
    V, d, ff, nb, N, T = 64, 64, 128, 2, 4, 40
    m = capture.TransformerModel(V, d, ff, nb, N, T, heads=2, seed=1)
    tokens, targets, _, _ = batch(V, N, T, dev)
    m.gradients(tokens, targets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.gradients(tokens, targets)
    tokens.copy_(batch(V, N, T, dev, 9)[0])
    graph.replay()
    tda.tda_device_status()
    got = [g.clone() for g in m.grads]
    m.gradients(tokens, targets)
    assert all(torch.equal(a, b) for a, b in zip(got, m.grads))


def test_command(dev, capsys):
    capture.main(["--attention"])
    out = capsys.readouterr().out
    assert "step 4" in out and "of 64 examples" in out
