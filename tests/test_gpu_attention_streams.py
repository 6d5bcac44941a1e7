"""Attention on another stream than the current one: everything allocated and filled first, the stream after it, and all of it
kept until the stream is done."""
import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild
from test_gpu_attention import BF, F32, KIND, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("mask,cap,buckets", [("docs", 20.0, 16), ("any", 0.0, 0), ("causal", 0.0, 16)])
def test_on_another_stream(dev, mask, cap, buckets, dtype):
    p = Problem(dev, 2, 300, 4, 2, 64, dtype, mask, cap, buckets, 64 if buckets else 0)
    p.forward()
    p.backward()
    want = [x.clone() for x in (p.O, p.lse, p.dQ, p.dK, p.dV) + ((p.dtable,) if buckets else ())]
    outs = [torch.full_like(x, 7.0) for x in want]
    O, lse, dQ, dK, dV = outs[:5]
    dtable = outs[5] if buckets else None
    ws = [torch.full((max(tda.tda_attention_workspace_size(op, p.L), 1),), 255, dtype=torch.uint8, device=dev)
          for op in (tda.TDA_ATTENTION_FORWARD, tda.TDA_ATTENTION_BACKWARD)]
    s = torch.cuda.Stream()
    ld = lambda x: x.stride(0)  # noqa: E731
    for _ in range(3):
        s.wait_stream(torch.cuda.current_stream())
        tda.tda_attention_forward(p.L, p.Q, ld(p.Q), p.K, ld(p.K), p.V, ld(p.V), p.range, p.bucket, p.table, None, O, ld(O), lse, ws[0],
                                  ws[0].numel(), s)
        tda.tda_attention_backward(p.L, p.Q, ld(p.Q), p.K, ld(p.K), p.V, ld(p.V), p.range, p.bucket, p.table, None, O, ld(O), lse, p.dO,
                                   ld(p.dO), dQ, ld(dQ), dK, ld(dK), dV, ld(dV), dtable, KIND[dtype], 0.0, ws[1], ws[1].numel(), s)
        s.synchronize()
        tda.tda_device_status()
        for got, exp in zip(outs, want):
            assert torch.equal(got, exp)
            got.fill_(7.0)
