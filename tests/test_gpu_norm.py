"""Root-mean-square norm and its backward pass against 64 bits. Tolerances: u = half a step of the output's type per
rounding (2^-8 bf16, 2^-24 fp32), 2^-24 per fp32 operation on the sums' magnitudes."""
import math

import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild

pytestmark = pytest.mark.gpu

KIND = {torch.float32: tda.TDA_F32, torch.bfloat16: tda.TDA_BF16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
D = torch.float64
EPS = 1e-5


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


def wide(rows, cols, gap, shift, dtype, dev, gen, fill=None):
    buf = torch.empty(rows * (cols + gap) + shift + 16, dtype=torch.float32, device=dev)
    buf = (buf.normal_(generator=gen) if fill is None else buf.fill_(fill)).to(dtype)
    return buf, buf[shift:shift + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]


def untouched(buf, rows, cols, gap, shift):
    assert (buf[:shift] == 7).all() and (buf[shift + rows * (cols + gap):] == 7).all()
    assert (buf[shift:shift + rows * (cols + gap)].view(rows, cols + gap)[:, cols:] == 7).all()


CASES = [
    # (M, d, gap, shift)
    (1, 1, 0, 0), (1, 64, 0, 0), (5, 7, 0, 1), (33, 512, 0, 0), (3, 513, 3, 0), (9, 1024, 8, 8), (130, 1000, 0, 0),
    (7, 1025, 0, 0), (64, 1363, 0, 0), (1000, 2048, 0, 0), (3, 4096, 8, 0), (257, 4100, 4, 4), (4, 16384, 0, 0),
    (3, 16392, 0, 0), (2, 32768, 0, 0), (2, 32767, 0, 0), (5000, 96, 0, 0), (2500, 1100, 0, 0),
]


@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CASES)
def test_norm(dev, case, dtype, residual):
    M, d, gap, shift = case
    gen = torch.Generator(device=dev).manual_seed(M + 3 * d)
    u = HALF[dtype]
    x, r = (wide(M, d, gap, shift, dtype, dev, gen)[1] for _ in range(2))
    if M > 2:
        x[1] = 0
        r[1] = 0  # padding
    w = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(dtype)
    hbuf, h = wide(M, d, gap, shift, dtype, dev, gen, fill=7.0)
    ybuf, y = wide(M, d, gap, shift, dtype, dev, gen, fill=7.0)
    rstd = torch.full((M + 1,), 7.0, device=dev)
    k = KIND[dtype]
    ld = d + gap
    tda.tda_rmsnorm_forward(k, x, ld, r if residual else None, ld, M, d, w, EPS, h if residual else None, ld, y, ld, rstd)
    tda.tda_device_status()
    stored = (x.to(D) + r.to(D)).to(torch.float32).to(dtype) if residual else x
    if residual:
        assert torch.equal(h, stored)
        untouched(hbuf, M, d, gap, shift)
    s = stored.to(D)
    want = 1 / torch.sqrt(s.square().mean(1) + EPS)
    e = 2.0 ** -24 * (d / 32 + 20)  # 32 values a thread and the joining, relative: all terms are positive
    assert ((rstd[:M].to(D) - want).abs() <= e * want).all() and rstd[M] == 7
    ref = s * want[:, None] * w.to(D)
    assert ((y.to(D) - ref).abs() <= (u + e) * ref.abs() + 1e-37).all()
    untouched(ybuf, M, d, gap, shift)
    # in place
    x2 = x.clone()
    tda.tda_rmsnorm_forward(k, x2, d, None, 0, M, d, w, EPS, None, 0, x2, d)
    y2 = torch.empty_like(x2)
    tda.tda_rmsnorm_forward(k, x, ld, None, 0, M, d, w, EPS, None, 0, y2, d)
    assert torch.equal(x2, y2)


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CASES)
def test_norm_backward(dev, case, dtype, residual, grad):
    if dtype == torch.float32 and grad == torch.bfloat16:
        return
    M, d, gap, shift = case
    gen = torch.Generator(device=dev).manual_seed(M + 5 * d)
    h, dy, dres = (wide(M, d, gap, shift, dtype, dev, gen)[1] for _ in range(3))
    if M > 2:
        dy[1] = 0
        h[1] = 0
    w = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(dtype)
    s = h.to(D)
    rstd = (1 / torch.sqrt(s.square().mean(1) + EPS)).float()
    buf, dx = wide(M, d, gap, shift, dtype, dev, gen, fill=7.0)
    dw0 = torch.randn(d, generator=gen, device=dev).to(grad)
    wsb = tda.tda_rmsnorm_workspace_size(M, d)
    ws = torch.full((wsb,), 255, dtype=torch.uint8, device=dev)
    ld, k = d + gap, KIND[dtype]
    n = s * rstd.to(D)[:, None]
    g = dy.to(D) * w.to(D)
    want_dx = rstd.to(D)[:, None] * (g - n * (g * n).mean(1, keepdim=True)) + (dres.to(D) if residual else 0)
    want_dw = (dy.to(D) * n).sum(0)
    mag = rstd.to(D)[:, None] * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
    tol_dx = HALF[dtype] * want_dx.abs() + 2.0 ** -24 * (d / 32 + 24) * mag + 2.0 ** -24 * want_dx.abs() + 1e-37
    for beta in (0.0, -0.5):
        dw = dw0.clone()
        tda.tda_rmsnorm_backward(k, h, ld, rstd, w, dy, ld, dres if residual else None, ld, M, d, dx, ld, dw, KIND[grad], beta, ws, wsb)
        tda.tda_device_status()
        assert ((dx.to(D) - want_dx).abs() <= tol_dx).all()
        ref = want_dw + beta * dw0.to(D)
        tol = HALF[grad] * ref.abs() + 2.0 ** -24 * (M + 8) * (dy.to(D) * n).abs().sum(0) + 2.0 ** -24 * dw0.to(D).abs() + 1e-37
        assert ((dw.to(D) - ref).abs() <= tol).all()
        untouched(buf, M, d, gap, shift)
        again = dw0.clone()
        tda.tda_rmsnorm_backward(k, h, ld, rstd, w, dy, ld, None, 0, M, d, None, 0, again, KIND[grad], beta, ws, wsb)
        assert torch.equal(again, dw)  # without dx, the same bits
    only = dy.clone()
    tda.tda_rmsnorm_backward(k, h, ld, rstd, w, only, d, dres if residual else None, ld, M, d, only, d)  # in place, no dw
    assert torch.equal(only, dx.contiguous()) or not torch.isfinite(only.float()).all()


def test_norm_other_streams_and_graphs(dev):
    x = torch.randn(300, 2048, device=dev).bfloat16()
    w = torch.ones(2048, device=dev).bfloat16()
    y, dx, rstd, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(300, device=dev), torch.empty(2048, device=dev)
    wsb = tda.tda_rmsnorm_workspace_size(300, 2048)
    ws = torch.empty(wsb, dtype=torch.uint8, device=dev)

    def both(stream=None):
        tda.tda_rmsnorm_forward(tda.TDA_BF16, x, 2048, None, 0, 300, 2048, w, EPS, None, 0, y, 2048, rstd, stream)
        tda.tda_rmsnorm_backward(tda.TDA_BF16, x, 2048, rstd, w, y, 2048, None, 0, 300, 2048, dx, 2048, dw, tda.TDA_F32, 0.0, ws,
                                 wsb, stream)
        return [t.clone() for t in (y, dx, dw)] if stream is None else None

    want = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    both(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, dw)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    x.mul_(-2)
    graph.replay()
    got = [t.clone() for t in (y, dx, dw)]
    assert all(torch.equal(a, b) for a, b in zip(got, both())) and not torch.equal(got[0], want[0])


def test_nan_stays_in_its_row(dev):
    x = torch.randn(40, 600, device=dev)
    x[3, 5], x[7, 9] = math.nan, math.inf
    w, y = torch.ones(600, device=dev), torch.empty(40, 600, device=dev)
    tda.tda_rmsnorm_forward(tda.TDA_F32, x, 600, None, 0, 40, 600, w, EPS, None, 0, y, 600)
    bad = ~torch.isfinite(y).all(1)
    assert bad[3] and bad[7] and bad.sum() == 2


@pytest.mark.parametrize("M,d", [(263000, 8192), (5000000, 8)])
def test_many_rows(dev, M, d):
    """Rows past 2^31 values, and millions of short ones; the last rows and the weight's gradient against 64 bits."""
    g = torch.Generator(device=dev).manual_seed(1)
    x = torch.randn((1000, d), generator=g, device=dev).bfloat16().repeat(M // 1000, 1)  # a thousand rows over and over
    dy, w = x.roll(1, 0), torch.randn(d, generator=g, device=dev).bfloat16()
    y, dx = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    rstd, dw = torch.empty(M, device=dev), torch.empty(d, device=dev)
    tda.tda_rmsnorm_forward(tda.TDA_BF16, x, d, None, 0, M, d, w, EPS, None, 0, y, d, rstd)
    wsb = tda.tda_rmsnorm_workspace_size(M, d)
    ws = torch.empty(wsb, dtype=torch.uint8, device=dev)
    tda.tda_rmsnorm_backward(tda.TDA_BF16, x, d, rstd, w, dy, d, None, 0, M, d, dx, d, dw, tda.TDA_F32, 0.0, ws, wsb)
    for out in (y, dx):  # equal rows give equal bits
        blocks = out.view(M // 1000, 1000, d)
        assert torch.equal(blocks[1:-1], blocks[1:2].expand(M // 1000 - 2, 1000, d)) and torch.equal(blocks[-1, 1:], blocks[1, 1:])
    a, b = x[-1000:].to(D), dy[-1000:].to(D)
    by = 1 / (a.square().mean(1, keepdim=True) + EPS).sqrt()
    n, gr = a * by, b * w.to(D)
    want = n * w.to(D)
    assert ((y[-1000:].to(D) - want).abs() <= (2.0 ** -8 + 8 * 2.0 ** -24) * want.abs()).all()
    s = (gr * n).mean(1, keepdim=True)
    want, size = by * (gr - n * s), by * (gr.abs() + n.abs() * (gr * n).abs().mean(1, keepdim=True))
    assert ((dx[-1000:].to(D) - want).abs() <= 2.0 ** -8 * want.abs() + 64 * 2.0 ** -24 * size).all()
    # every row has all others' terms in its column; a CTA adds up to M / 152 rows one after the other, then 608 shares
    total, size = (b * n).sum(0) * (M // 1000), (b * n).abs().sum(0) * (M // 1000)
    assert ((dw.to(D) - total).abs() <= (M / 152 + 608) * 2.0 ** -24 * size).all()
