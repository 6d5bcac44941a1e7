"""The first calls of a process, captured at once; and the backward pass without the bias's gradient."""
import subprocess
import sys
import textwrap

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


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_first_call_in_a_capture(dev, dtype):
    code = f"""
        import torch
        import paper_2609_38767_gb300 as tda
        N, T, H, KV, hd, dt = 2, 200, 4, 2, 64, torch.{dtype}
        kind = tda.TDA_BF16 if dt == torch.bfloat16 else tda.TDA_F32
        M, a, b = N * T, H * hd, KV * hd
        g = torch.Generator(device="cuda").manual_seed(1)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)
        Q, K, V, dO, x, w, table = rand(M, a), rand(M, b), rand(M, b), rand(M, a), rand(M, a), rand(a), rand(8, H)
        O, dQ, dK, dV, y, dx = (torch.empty_like(t) for t in (Q, Q, K, V, x, x))
        lse, rstd, dw = torch.empty((N, H, T), device="cuda"), torch.empty(M, device="cuda"), torch.empty(a, device="cuda")
        dtable, ranges = torch.empty((8, H), device="cuda"), torch.empty((N, T, 2), dtype=torch.int32, device="cuda")
        doc = (torch.arange(T, device="cuda") // 60).int().repeat(N, 1)
        bucket = torch.empty(41, dtype=torch.int32)
        tda.tda_position_buckets(8, 20, False, bucket)
        bucket = bucket.cuda()
        L = tda.AttentionDesc(N, T, H, KV, hd, kind, cap=20.0, n_buckets=8, max_distance=20)
        size = max([tda.tda_attention_workspace_size(op, L) for op in (0, 1)] + [tda.tda_rmsnorm_workspace_size(M, a)])
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")

        def step():
            tda.tda_attention_ranges(N, T, doc, None, True, 0, ranges)
            tda.tda_rmsnorm_forward(kind, x, a, None, 0, M, a, w, 1e-5, None, 0, y, a, rstd)
            tda.tda_attention_forward(L, Q, a, K, b, V, b, ranges, bucket, table, None, O, a, lse, ws, size)
            tda.tda_attention_backward(L, Q, a, K, b, V, b, ranges, bucket, table, None, O, a, lse, dO, a, dQ, a, dK, b, dV, b, dtable,
                                       tda.TDA_F32, 0.0, ws, size)
            tda.tda_rmsnorm_backward(kind, x, a, rstd, w, dO, a, None, 0, M, a, dx, a, dw, tda.TDA_F32, 0.0, ws, size)

        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        outs = (ranges, y, rstd, O, lse, dQ, dK, dV, dtable, dx, dw)
        for t in outs:
            t.fill_(7)
        graph.replay()
        got = [t.clone() for t in outs]
        step()
        tda.tda_device_status()
        assert all(torch.equal(p, q) for p, q in zip(got, outs))
        print("equal")
    """
    out = subprocess.run([sys.executable, "-c", textwrap.dedent(code)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip().endswith("equal"), out.stdout + out.stderr


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("mask,cap,slope", [("docs", 20.0, False), ("causal", 0.0, True)])
def test_without_the_bias_gradient(dev, mask, cap, slope, dtype):
    """dtable NULL with a bias: the other gradients' bits stay."""
    p = Problem(dev, 2, 300, 4, 2, 64, dtype, mask, cap, 12, 64, slope)
    p.forward()
    p.backward()
    outs = [torch.full_like(x, 7.0) for x in (p.dQ, p.dK, p.dV)]
    dQ, dK, dV = outs
    wsb = tda.tda_attention_workspace_size(tda.TDA_ATTENTION_BACKWARD, p.L)
    ws = torch.full((wsb,), 255, dtype=torch.uint8, device=dev)
    ld = lambda x: x.stride(0)  # noqa: E731
    tda.tda_attention_backward(p.L, p.Q, ld(p.Q), p.K, ld(p.K), p.V, ld(p.V), p.range, p.bucket, p.table, p.slope, p.O, ld(p.O), p.lse, p.dO,
                               ld(p.dO), dQ, ld(dQ), dK, ld(dK), dV, ld(dV), None, KIND[dtype], 0.0, ws, wsb)
    tda.tda_device_status()
    assert all(torch.equal(x, y) for x, y in zip(outs, (p.dQ, p.dK, p.dV)))
