"""A million examples of one token, past 2^31 values and with a tile of its own for every token and head: a token with one key has that
key's value, to the last bit, and gradients only through it."""
import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild
from test_gpu_attention import BF, F32, KIND

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    yield torch.device("cuda:0")
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,cap,ranged", [(BF, 0.0, False), (BF, 30.0, True), (F32, 0.0, True)])
def test_a_million_examples(dev, dtype, cap, ranged):
    N, H, hd = (1 << 20) + 3, 32, 64
    L = tda.AttentionDesc(N, 1, H, 1, hd, KIND[dtype], cap=cap)
    gen = torch.Generator(device=dev).manual_seed(5)
    a = H * hd
    Q = torch.randn((1024, a), generator=gen, device=dev).to(dtype).repeat(N // 1024 + 1, 1)[:N]
    K, V = (torch.randn((N, hd), generator=gen, device=dev).to(dtype) for _ in range(2))
    rng = None
    if ranged:  # every 5th token sees nothing
        rng = torch.zeros((N, 1, 2), dtype=torch.int32, device=dev)
        rng[:, 0, 1] = (torch.arange(N, device=dev) % 5 != 0).int()
    live = torch.ones(N, dtype=torch.bool, device=dev) if rng is None else rng[:, 0, 1] > 0
    O = torch.full((N, a), 7.0, dtype=dtype, device=dev)
    lse = torch.full((N, H, 1), 7.0, device=dev)
    sizes = [tda.tda_attention_workspace_size(op, L) for op in (tda.TDA_ATTENTION_FORWARD, tda.TDA_ATTENTION_BACKWARD)]
    ws = torch.empty(max(sizes[0], 1), dtype=torch.uint8, device=dev)
    tda.tda_attention_forward(L, Q, a, K, hd, V, hd, rng, None, None, None, O, a, lse, ws, sizes[0])
    tda.tda_device_status()
    want = torch.where(live[:, None], V, torch.zeros_like(V))
    for h in range(H):
        assert torch.equal(O[:, h * hd:(h + 1) * hd], want)
    assert torch.equal(torch.isinf(lse[:, :, 0]), ~live[:, None].expand(N, H))
    if dtype == F32:
        return
    ws = torch.empty(sizes[1], dtype=torch.uint8, device=dev)
    dO = Q.flip(1)
    dQ = torch.full_like(Q, 7.0)
    dK, dV = torch.full_like(K, 7.0), torch.full_like(V, 7.0)
    tda.tda_attention_backward(L, Q, a, K, hd, V, hd, rng, None, None, None, O, a, lse, dO, a, dQ, a, dK, hd, dV, hd, None, tda.TDA_F32, 0.0,
                               ws, sizes[1])
    tda.tda_device_status()
    assert (dQ == 0).all() and (dK == 0).all()
    heads = dO[:1024].double().view(1024, H, hd)  # rows repeat
    total, size = heads.sum(1), heads.abs().sum(1)
    total, size = (x.repeat(N // 1024 + 1, 1)[:N] * live[:, None] for x in (total, size))
    # P is 1 as bf16 (off by 2^-21 of the score, the cap and lse before); fp32 sums of 32 products, rounded once
    assert ((dV.double() - total).abs() <= 2.0 ** -8 * total.abs() + 2.0 ** -15 * size).all()
