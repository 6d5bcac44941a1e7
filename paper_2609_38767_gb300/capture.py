"""One training step of a small token model whose linears are then attributed.

The attribution calls take a layer's factors: its input A and the gradient B of the
loss by its output (Eq. 1). Here they are made with the library itself, as a
training program would: tokens are looked up (tda_embedding_forward), pass through
residual blocks h + W_down act(W_up h) of linear layers (tda_linear_forward, the
activation, bias and residual in the product's epilogue) and a linear head; the
backward pass leaves every linear's B beside its weight gradients
(tda_linear_backward), the table's gradient (tda_embedding_backward), and the whole
gradient is clipped to a global norm (tda_grad_clip) before the update. The X and B
that the step left are projected as they lie, [N][T][d] (tda_project), and scored.

    python -m paper_2609_38767_gb300.capture     # a few steps, then the examples that moved a query

The features are those of the gradient before clipping: the clipping scales the step's whole gradient, and so all its
examples' features, by one number. The loss (a softmax over the vocabulary), the sum of the two gradients that meet at
a residual and the update are torch operations.
"""
from __future__ import annotations

import math

import torch

import paper_2609_38767_gb300 as tda

_INDEX = {torch.int32: tda.TDA_I32, torch.int64: tda.TDA_I64}


class _Linear:
    """Weights, gradients and the step's tensors of one linear over M tokens."""

    def __init__(self, d_in, d_out, act, dtype, M, gen, device):
        kind = tda.TDA_BF16 if dtype == torch.bfloat16 else tda.TDA_F32
        self.L = tda.LinearDesc(d_in, d_out, act, kind)
        self.W = (torch.randn((d_out, d_in), generator=gen, device=device) / math.sqrt(d_in)).to(dtype)
        self.b = torch.zeros(d_out, dtype=dtype, device=device)
        self.dW = torch.empty((d_out, d_in), dtype=torch.float32, device=device)
        self.db = torch.empty(d_out, dtype=torch.float32, device=device)
        self.Z = torch.empty((M, d_out), dtype=dtype, device=device) if act != tda.TDA_ACT_NONE else None
        self.Y = torch.empty((M, d_out), dtype=dtype, device=device)
        self.B = torch.empty((M, d_out), dtype=dtype, device=device)
        self.X = None

    def forward(self, X, M, residual, ws):
        self.X = X
        di, do = self.L.d_in, self.L.d_out
        tda.tda_linear_forward(self.L, X, di, M, self.W, di, self.b, residual, do, self.Y, do, self.Z, do, ws, ws.numel())
        return self.Y

    def backward(self, dY, M, dX, ws):
        di, do = self.L.d_in, self.L.d_out
        tda.tda_linear_backward(self.L, dY, do, self.Z, do, M, self.X, di, self.W, di, self.B, do, dX, di, self.dW, di,
                                self.db, tda.TDA_F32, 0.0, ws, ws.numel())


class TokenModel:
    """Embedding, n_blocks residual blocks and a head, for batches of N examples of T tokens."""

    def __init__(self, vocab, d, ff, n_blocks, N, T, *, dtype=torch.bfloat16, act=tda.TDA_ACT_SILU, max_norm=1.0,
                 lr=0.1, seed=0, device="cuda"):
        self.V, self.d, self.N, self.T, self.M = vocab, d, N, T, N * T
        self.dtype, self.kind, self.max_norm, self.lr = dtype, tda.TDA_BF16 if dtype == torch.bfloat16 else tda.TDA_F32, max_norm, lr
        gen = torch.Generator(device=device).manual_seed(seed)
        self.scale = math.sqrt(d)
        self.E = (torch.randn((vocab, d), generator=gen, device=device) / math.sqrt(d)).to(dtype)
        self.dE = torch.empty((vocab, d), dtype=torch.float32, device=device)
        mk = lambda di, do, a: _Linear(di, do, a, dtype, self.M, gen, device)  # noqa: E731
        self.blocks = [(mk(d, ff, act), mk(ff, d, tda.TDA_ACT_NONE)) for _ in range(n_blocks)]
        self.head = mk(d, vocab, tda.TDA_ACT_NONE)
        self.linears = [x for b in self.blocks for x in b] + [self.head]
        self.h0 = torch.empty((self.M, d), dtype=dtype, device=device)
        self.dh = [torch.empty((self.M, d), dtype=dtype, device=device) for _ in range(2)]
        self.du = torch.empty((self.M, ff), dtype=dtype, device=device)
        grads = [self.dE] + [g for x in self.linears for g in (x.dW, x.db)]
        self.params = [self.E] + [p for x in self.linears for p in (x.W, x.b)]
        self.grads, self.refs = grads, tda.tensor_list(grads)
        self.norm = torch.empty(1, dtype=torch.float32, device=device)
        need = max([tda.tda_embedding_workspace_size(vocab, d, self.M),
                    tda.tda_grad_clip_workspace_size(self.refs, len(grads))]
                   + [tda.tda_linear_workspace_size(tda.TDA_LINEAR_BACKWARD, x.L, self.M) for x in self.linears])
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)

    def forward(self, tokens):
        """Logits [M][V] of tokens [N][T] (int32 or int64, on the model's device; a negative id is padding)."""
        if tokens.dtype not in _INDEX or tokens.numel() != self.M or tokens.device != self.E.device:
            raise ValueError(f"tokens are {self.N} x {self.T} int32 or int64 ids on {self.E.device}, not "
                             f"{tuple(tokens.shape)} {tokens.dtype} on {tokens.device}")
        self.tokens, self.index = tokens.reshape(-1).contiguous(), _INDEX[tokens.dtype]
        tda.tda_embedding_forward(self.kind, self.E, self.d, self.V, self.d, self.index, self.tokens, self.M, self.scale,
                                  self.h0, self.d)
        h = self.h0
        for up, down in self.blocks:
            h = down.forward(up.forward(h, self.M, None, self.ws), self.M, h, self.ws)
        return self.head.forward(h, self.M, None, self.ws)

    def backward(self, dlogits):
        """Gradients of every parameter and every linear's B, from dlogits [M][V] of the model's type (zero rows for
        padding)."""
        if (tuple(dlogits.shape) != (self.M, self.V) or dlogits.dtype != self.dtype or dlogits.device != self.E.device
                or not dlogits.is_contiguous()):
            raise ValueError(f"dlogits are contiguous {self.M} x {self.V} {self.dtype} on {self.E.device}")
        dh, other = self.dh
        self.head.backward(dlogits, self.M, dh, self.ws)
        for up, down in reversed(self.blocks):
            down.backward(dh, self.M, self.du, self.ws)
            up.backward(self.du, self.M, other, self.ws)
            other += dh  # the residual's share of the gradient
            dh, other = other, dh
        tda.tda_embedding_backward(self.kind, dh, self.d, self.V, self.d, self.index, self.tokens, self.M, self.scale,
                                   tda.TDA_F32, self.dE, self.d, 0.0, self.ws, self.ws.numel())

    def loss_gradient(self, logits, targets):
        """Mean cross entropy over each example's live tokens, summed over the batch, and its gradient: a
        softmax less the target; positions with a negative target are padding."""
        t = targets.reshape(-1).long()
        live = (t >= 0).float().unsqueeze(1)
        z = logits.float()
        z = z - z.amax(1, keepdim=True)
        lse = z.exp().sum(1, keepdim=True).log()
        per = live / live.view(self.N, self.T).sum(1).clamp(min=1).repeat_interleave(self.T).unsqueeze(1)
        at = t.clamp(min=0).unsqueeze(1)
        loss = ((lse - z.gather(1, at)) * per).sum()
        g = (z - lse).exp()
        g.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
        return loss, (g * per).to(self.dtype)

    def gradients(self, tokens, targets):
        loss, dlogits = self.loss_gradient(self.forward(tokens), targets)
        self.backward(dlogits)
        return loss

    def step(self, tokens, targets):
        """One clipped gradient step; returns (loss, gradient norm before clipping) as device tensors."""
        loss = self.gradients(tokens, targets)
        tda.tda_grad_clip(self.refs, len(self.grads), self.max_norm, self.norm, self.ws, self.ws.numel())
        for p, g in zip(self.params, self.grads):
            p.add_(g.to(p.dtype), alpha=-self.lr)
        return loss, self.norm

    def features(self, k, seed=0):
        """Projected per-example gradients [N][linears * k * k] of the last backward pass, from its factors as they lie."""
        D, nl = k * k, len(self.linears)
        phi = torch.empty((self.N, nl * D), dtype=torch.float32, device=self.E.device)
        for i, x in enumerate(self.linears):
            L = tda.LayerDesc(x.L.d_in, x.L.d_out, self.T, k, k, seed=seed, layer=i)
            tda.tda_project(L, self.kind, x.X, x.B, self.N, phi[:, i * D:], nl * D, tda.TDA_ROUTE_FACTORED)
        return phi


def main():
    torch.manual_seed(0)
    V, N, T, k = 512, 64, 32, 16
    m = TokenModel(V, d=128, ff=256, n_blocks=2, N=N, T=T)
    # every example repeats a short pattern of its own; examples 2 i and 2 i + 1 share it
    pattern = torch.randint(0, V, (N // 2, 4), device="cuda").repeat_interleave(2, 0)
    seq = pattern.repeat(1, T // 4 + 1)
    tokens, targets = seq[:, :T].int().contiguous(), seq[:, 1:T + 1].int().contiguous()
    tokens[:, -3:], targets[:, -3:] = -1, -1  # padding
    for i in range(5):
        loss, norm = m.step(tokens, targets)
        print(f"step {i}: loss {float(loss) / N:.4f} per example, gradient norm {float(norm):.3f}")
    m.gradients(tokens, targets)
    phi = m.features(k)
    DT = phi.shape[1]
    S = torch.empty((N, N), device="cuda")
    tda.tda_score(phi, tda.TDA_F32, N, DT, phi, N, DT, DT, S, N)
    S.fill_diagonal_(float("-inf"))
    idx = torch.empty((N, 1), dtype=torch.int32, device="cuda")
    tda.tda_topk(S, N, N, N, 1, idx)
    tda.tda_device_status()
    twin = torch.arange(N, device="cuda") ^ 1
    print(f"{int((idx[:, 0] == twin).sum())} of {N} examples have their twin as the most influential other one")


if __name__ == "__main__":
    main()
