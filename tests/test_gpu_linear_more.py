"""The linear layer, further: launches that follow each other closely, values at the edges of the activations, long sums,
several threads. Plain fp64 implementations as in test_gpu_linear.py, whose derived bounds hold here too."""
import math

import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild

pytestmark = pytest.mark.gpu

F64 = torch.float64
KIND = {torch.float32: tda.TDA_F32, torch.bfloat16: tda.TDA_BF16}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


def workspace(op, L, M, dev):
    wsb = tda.tda_linear_workspace_size(op, L, M)
    return torch.full((max(wsb, 1),), 0x7F, dtype=torch.uint8, device=dev), wsb


def test_launches_close_together_repeat_bit_for_bit(dev):
    """Calls of one or a few tiles per SM pair queued without a pause: each CTA starts where another has just left, so a
    signal or a copy that outlives its CTA would land in the next one's shared memory."""
    gen = torch.Generator(device=dev).manual_seed(21)
    jobs = []
    for M, di, do, dtype in ((512, 256, 1024, torch.bfloat16), (2048, 128, 2304, torch.bfloat16),
                             (1024, 192, 1280, torch.float32), (4096, 64, 5120, torch.bfloat16)):
        mk = lambda *s: torch.randn(s, generator=gen, device=dev).to(dtype)
        L = tda.LinearDesc(di, do, tda.TDA_ACT_NONE, KIND[dtype])
        ws, wsb = workspace(tda.TDA_LINEAR_BACKWARD, L, M, dev)
        jobs.append((L, M, di, do, mk(M, di), mk(do, di), mk(M, do), ws, wsb))

    def run(j):
        L, M, di, do, X, W, dY, ws, wsb = j
        Y, dX, dW = torch.empty_like(dY), torch.empty_like(X), torch.empty((do, di), device=dev)
        tda.tda_linear_forward(L, X, di, M, W, di, None, None, 0, Y, do, None, 0, ws, wsb)
        tda.tda_linear_backward(L, dY, do, None, 0, M, X, di, W, di, None, 0, dX, di, dW, di, None, tda.TDA_F32, 0.0, ws, wsb)
        return Y, dX, dW

    first = [run(j) for j in jobs]
    wrong = torch.zeros(1, dtype=torch.int64, device=dev)
    for _ in range(40):
        got = [run(j) for j in jobs]
        for a, b in zip(first, got):
            for x, y in zip(a, b):
                wrong += (x != y).sum()
    tda.tda_device_status()
    assert int(wrong) == 0
    for (L, M, di, do, X, W, *_), (Y, _, _) in zip(jobs, first):
        ref = X.to(F64) @ W.to(F64).t()
        assert float((Y.to(F64) - ref).norm() / ref.norm()) <= (2.4e-3 if X.dtype == torch.bfloat16 else 1e-6)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [1, 40, 2048])
def test_infinite_pre_activations(dev, M, act, dtype):
    """Infinities that enter by the bias, through each kernel: +inf passes every activation, -inf leaves relu as 0 and the
    others not finite; the slopes are the limits 1 and 0 (below 2^-20, the functions' own error)."""
    di, do = 64, 1024
    gen = torch.Generator(device=dev).manual_seed(31)
    mk = lambda *s: torch.randn(s, generator=gen, device=dev).to(dtype)
    X, W, b, dY = mk(M, di), mk(do, di), mk(do), mk(M, do)
    up, down = torch.arange(3, do, 29, device=dev), torch.arange(5, do, 31, device=dev)
    up = up[~torch.isin(up, down)]
    rest = torch.ones(do, dtype=torch.bool, device=dev)
    rest[up] = rest[down] = False
    b[up], b[down] = float("inf"), float("-inf")
    L = tda.LinearDesc(di, do, ACTS.index(act), KIND[dtype])
    ws, wsb = workspace(tda.TDA_LINEAR_BACKWARD, L, M, dev)
    Y, Z, B = torch.empty_like(dY), torch.empty_like(dY), torch.empty_like(dY)
    tda.tda_linear_forward(L, X, di, M, W, di, b, None, 0, Y, do, Z, do, ws, wsb)
    tda.tda_linear_backward(L, dY, do, Z, do, M, None, 0, None, 0, B, do, None, 0, None, 0, None, tda.TDA_F32, 0.0, ws, wsb)
    tda.tda_device_status()
    inf = float("inf")
    assert bool((Z[:, up] == inf).all()) and bool((Z[:, down] == -inf).all())
    assert bool((Y[:, up] == inf).all())
    assert bool((Y[:, down] == 0).all() if act == "relu" else ~torch.isfinite(Y[:, down]).any())
    assert bool(torch.isfinite(Y[:, rest]).all()) and bool(torch.isfinite(B).all())
    limit = dY.clone()
    if act != "none":
        limit[:, down] = 0
    off = (B - limit).to(F64).abs()
    for cols in (up, down):
        assert bool((off[:, cols] <= 2.0 ** -20 * dY[:, cols].to(F64).abs()).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M", [1, 24, 1024])
def test_activation_tails_are_right_in_proportion(dev, M, act, dtype):
    """W = I, z from -1 down to where the value leaves the normal numbers. bf16: 2^-11 for the functions and half an ulp
    (2^-8); fp32: the exponential's argument (up to 88) is rounded a few times, 4 * 88 * 2^-24 < 2^-15 of the value."""
    d = 512
    z = torch.linspace(-1, -88 if act == "silu" else -13, M * d, dtype=F64).view(M, d).to(device=dev).to(dtype)
    L = tda.LinearDesc(d, d, ACTS.index(act), KIND[dtype])
    ws, wsb = workspace(tda.TDA_LINEAR_FORWARD, L, M, dev)
    Y, Z = torch.empty_like(z), torch.empty_like(z)
    tda.tda_linear_forward(L, z, d, M, torch.eye(d, device=dev).to(dtype), d, None, None, 0, Y, d, Z, d, ws, wsb)
    tda.tda_device_status()
    assert torch.equal(Z, z) or dtype == torch.float32
    x = Z.to(F64)
    if act == "gelu":
        # z Phi(z) by the scaled function, which keeps the tail's digits
        ref = x * 0.5 * torch.special.erfcx(-x / math.sqrt(2)) * torch.exp(-0.5 * x * x)
    elif act == "gelu_tanh":
        ref = x / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    else:
        ref = x / (1 + torch.exp(-x))
    held = ref.abs() >= 1e-36
    off = ((Y.to(F64) - ref).abs() / ref.abs())[held]
    assert int(held.sum()) > 0.6 * held.numel()
    assert float(off.max()) <= (2.0 ** -8 + 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -15), float(off.max())


def test_first_call_of_a_host_thread(dev):
    """A thread that has done no CUDA work yet calls the library: its tensor maps need a context too. Every buffer is made
    beforehand, so that the call is the thread's first."""
    import threading

    mk = lambda *s: torch.randn(s, device=dev).bfloat16()
    s = torch.cuda.current_stream().cuda_stream
    calls = []
    for M, di, do in ((2048, 256, 2304), (300, 256, 520)):
        L = tda.LinearDesc(di, do, tda.TDA_ACT_NONE, tda.TDA_BF16)
        X, W, Y, dX, dW = mk(M, di), mk(do, di), mk(M, do), mk(M, di), torch.zeros((do, di), device=dev)
        calls.append((lambda L=L, M=M, di=di, do=do, X=X, W=W, Y=Y: tda.tda_linear_forward(
            L, X, di, M, W, di, None, None, 0, Y, do, stream=s), Y))
        dY = mk(M, do)
        calls.append((lambda L=L, M=M, di=di, do=do, X=X, W=W, dY=dY, dX=dX, dW=dW: tda.tda_linear_backward(
            L, dY, do, None, 0, M, X, di, W, di, None, 0, dX, di, dW, di, None, tda.TDA_F32, 0.0, None, 0, stream=s), dW))
    N, T, d, k = 8, 128, 256, 32
    A, B, phi = mk(N, T, d), mk(N, T, d), torch.zeros((N, k * k), device=dev)
    P = tda.LayerDesc(d, d, T, k, k)
    calls.append((lambda: tda.tda_project(P, tda.TDA_BF16, A, B, N, phi, k * k, tda.TDA_ROUTE_FACTORED, stream=s), phi))
    Q, F, S = torch.randn(64, 1024, device=dev), torch.randn(256, 1024, device=dev), torch.zeros(64, 256, device=dev)
    calls.append((lambda: tda.tda_score(Q, tda.TDA_F32, 64, 1024, F, 256, 1024, 1024, S, 256, stream=s), S))
    for call, out in calls:
        call()
        want = out.clone()
        out.zero_()
        torch.cuda.synchronize()
        failed = []

        def first(call=call, failed=failed):
            try:
                call()
            except Exception as e:  # noqa: BLE001
                failed.append(e)

        t = threading.Thread(target=first)
        t.start()
        t.join()
        assert not failed, failed
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    tda.tda_device_status()


def test_threads_with_streams_and_workspaces_of_their_own(dev):
    """Four host threads at once, each on its stream: the same bits as one after the other."""
    import threading

    jobs = []
    for k, (M, di, do, dtype) in enumerate(((700, 264, 1000, torch.bfloat16), (2048, 512, 2304, torch.bfloat16),
                                            (333, 130, 520, torch.float32), (9, 1024, 640, torch.float32))):
        gen = torch.Generator(device=dev).manual_seed(50 + k)
        mk = lambda *s: torch.randn(s, generator=gen, device=dev).to(dtype)
        L = tda.LinearDesc(di, do, tda.TDA_ACT_GELU_TANH, KIND[dtype])
        ws, wsb = workspace(tda.TDA_LINEAR_BACKWARD | tda.TDA_LINEAR_ANY_STRIDE, L, M, dev)
        jobs.append((L, M, di, do, mk(M, di), mk(do, di), mk(do), mk(M, do), ws, wsb))

    def run(j, stream):
        L, M, di, do, X, W, b, dY, ws, wsb = j
        with torch.cuda.stream(stream):
            Y, Z, B, dX = torch.empty_like(dY), torch.empty_like(dY), torch.empty_like(dY), torch.empty_like(X)
            dW, db = torch.empty((do, di), device=dev), torch.empty(do, device=dev)
            tda.tda_linear_forward(L, X, di, M, W, di, b, None, 0, Y, do, Z, do, ws, wsb)
            tda.tda_linear_backward(L, dY, do, Z, do, M, X, di, W, di, B, do, dX, di, dW, di, db, tda.TDA_F32, 0.0, ws, wsb)
        return Y, Z, B, dX, dW, db

    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    alone = [run(j, s) for j, s in zip(jobs, streams)]
    torch.cuda.synchronize()
    got, failed = [[] for _ in jobs], []

    def work(i):
        try:
            got[i] += [run(jobs[i], streams[i]) for _ in range(25)]
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    tda.tda_device_status()
    assert not failed
    for a, runs in zip(alone, got):
        assert len(runs) == 25 and all(torch.equal(x, y) for r in runs for x, y in zip(a, r))


@pytest.mark.parametrize("M", [4095, 4160, 20011, 70000])
@pytest.mark.parametrize("di,do", [(64, 128), (264, 520), (2048, 2304), (1801, 2563)])
def test_long_sums_of_one_sign_do_not_drift(dev, M, di, do):
    """fp32 dW of bf16 layers from operands of one sign. The tensor pipe adds 16 products at a time with truncation, at most
    2^-22 of the running sum, for 4096 tokens; what comes then is added with rounding, 2^-24 a time:
    256 * 2^-22 + (M / 4096 + 2) * 2^-24. Truncation on average takes half of a step of a sum that is half as
    large: no more than a quarter of the first term in the mean, which is what would grow with M."""
    gen = torch.Generator(device=dev).manual_seed(M + di)
    X = (torch.rand((M, di), generator=gen, device=dev) + 0.5).bfloat16()
    dY = (torch.rand((M, do), generator=gen, device=dev) + 0.5).bfloat16()
    W = torch.randn((do, di), generator=gen, device=dev).bfloat16()
    old = torch.rand((do, di), generator=gen, device=dev) * M
    L = tda.LinearDesc(di, do, tda.TDA_ACT_NONE, tda.TDA_BF16)
    ws, wsb = workspace(tda.TDA_LINEAR_BACKWARD, L, M, dev)
    ref = torch.zeros((do, di), dtype=F64, device=dev)
    for m in range(0, M, 8192):
        ref += dY[m:m + 8192].to(F64).t() @ X[m:m + 8192].to(F64)
    pipe, rnd = 256 * 2.0 ** -22, (M / 4096 + 2) * 2.0 ** -24
    for with_dx, beta in ((False, 0.0), (True, 0.0), (True, 1.0)):
        dX, dW = torch.empty_like(X), old.clone()
        tda.tda_linear_backward(L, dY, do, None, 0, M, X, di, W, di, None, 0, dX if with_dx else None, di, dW, di, None,
                                tda.TDA_F32, beta, ws, wsb)
        tda.tda_device_status()
        want = ref + beta * old.to(F64)
        off = (dW.to(F64) - want) / want
        assert float(off.abs().max()) <= pipe + rnd, float(off.abs().max())
        assert abs(float(off.mean())) <= pipe / 4 + rnd, float(off.mean())
        if with_dx:
            dx = dY.to(F64) @ W.to(F64)
            assert float((dX.to(F64) - dx).norm() / dx.norm()) <= 2.4e-3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,di,do", [(1, 16384, 520), (4, 8192, 264), (16, 20001, 130), (33, 14336, 1000), (300, 16384, 392),
                                     (1100, 8200, 2056)])
def test_long_rows(dev, M, di, do, dtype):
    """Sums over 8192 and more inputs, through each kernel, and dX over as many outputs. Bounds of test_gpu_linear.py: bf16
    (K / 16 + 16) 2^-22 of the sum of |products|, fp32 24 * 2^-22 + (6 K / 256 + 8) 2^-24, few fp32 rows a chain
    of K / 32 additions; then half an ulp."""
    gen = torch.Generator(device=dev).manual_seed(di + M)
    mk = lambda *s: torch.randn(s, generator=gen, device=dev).to(dtype)
    X, W, b = mk(M, di), (mk(do, di).float() / math.sqrt(di)).to(dtype), mk(do)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24

    def bound(K):
        if dtype == torch.bfloat16:
            return (K / 16 + 16) * 2.0 ** -22
        return max(24 * 2.0 ** -22 + (6 * K / 256 + 8) * 2.0 ** -24, (K / 32 + 8) * 2.0 ** -24)

    def check(got, ref, size, K):
        t = bound(K) * size + 2.0 ** -23 * size
        off = (got.to(F64) - ref).abs()
        assert bool((off <= t + half * (ref.abs() + t)).all()), float((off / size).max())
        assert float(off.norm() / ref.norm()) <= (2.4e-3 if dtype == torch.bfloat16 else 1.5e-6)

    L = tda.LinearDesc(di, do, tda.TDA_ACT_NONE, KIND[dtype])
    ws, wsb = workspace(tda.TDA_LINEAR_BACKWARD, L, M, dev)
    Y = torch.empty((M, do), dtype=dtype, device=dev)
    tda.tda_linear_forward(L, X, di, M, W, di, b, None, 0, Y, do, None, 0, ws, wsb)
    tda.tda_device_status()
    check(Y, X.to(F64) @ W.to(F64).t() + b.to(F64), X.to(F64).abs() @ W.to(F64).abs().t() + b.to(F64).abs(), di)
    # the transposed layer: di outputs, dX sums over them
    Wt, T = W.t().contiguous(), tda.LinearDesc(do, di, tda.TDA_ACT_NONE, KIND[dtype])
    ws, wsb = workspace(tda.TDA_LINEAR_BACKWARD, T, M, dev)
    dX = torch.empty((M, do), dtype=dtype, device=dev)
    tda.tda_linear_backward(T, X, di, None, 0, M, None, 0, Wt, do, None, 0, dX, do, None, 0, None, tda.TDA_F32, 0.0, ws, wsb)
    tda.tda_device_status()
    check(dX, X.to(F64) @ W.to(F64).t(), X.to(F64).abs() @ W.to(F64).abs().t(), di)
