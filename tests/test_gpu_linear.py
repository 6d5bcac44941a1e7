"""The linear layer (bias, activation, residual in the epilogue) and its backward pass against plain fp64
implementations: one token to thousands, odd widths, strides and alignments, every activation and type.

Tolerances from the arithmetic, S = sum of |products|: the tensor pipe adds 16 products at a time with truncation,
at most 2^-22 of the running magnitude each (fp32 operands: runs of 16 such additions, then rounding, and products
good to 2^-22); outputs are rounded once, half an ulp; the functions are good to 2^-20 where they are of size 1.
Beside these worst cases the Frobenius error is held to the size of the roundings taken at random."""
import math

import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
KIND = {torch.float32: tda.TDA_F32, torch.bfloat16: tda.TDA_BF16}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
F64 = torch.float64


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


def act64(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z * 1.0


def slope64(name, z):
    if name == "relu":
        return (z > 0).to(F64)
    z = z.clone().requires_grad_(True)
    return torch.autograd.grad(act64(name, z).sum(), z)[0]


def rows(gen, n, d, gap, shift, sigma, dtype, dev, fill=None):
    buf = torch.empty(n * (d + gap) + shift + 16, dtype=torch.float32, device=dev)
    buf = (buf.normal_(0, sigma, generator=gen) if fill is None else buf.fill_(fill)).to(dtype)
    return buf, buf[shift:shift + n * (d + gap)].view(n, d + gap)[:, :d]


def ws_for(op, L, M, dev, any_stride):
    wsb = tda.tda_linear_workspace_size(op | (tda.TDA_LINEAR_ANY_STRIDE if any_stride else 0), L, M)
    return torch.full((max(wsb, 1),), 0x7F, dtype=torch.uint8, device=dev), wsb


def product_bound(K, dtype):
    """Error of a K-long product as a share of S."""
    if dtype == torch.float32:
        return 24 * 2.0 ** -22 + (6 * K / 256 + 8) * U
    return (K / 16 + 16) * 2.0 ** -22


def close(got, ref, tol, fro=None):
    err = (got.to(F64) - ref).abs()
    assert bool(torch.isfinite(got.to(F64)).all())
    assert bool((err <= tol).all()), (float((err - tol).max()), float(err.max()))
    if fro is not None and ref.numel() >= 1000:  # enough values for a mean
        assert float(err.norm() / ref.norm()) <= fro, float(err.norm() / ref.norm())


def beside(buf, view_rows, d, gap, shift, value):
    inside = torch.zeros(buf.numel(), dtype=torch.bool, device=buf.device)
    inside[shift:shift + view_rows * (d + gap)].view(view_rows, d + gap)[:, :d] = True
    assert bool((buf[~inside] == value).all())


SHAPES = [
    # (M, d_in, d_out, gap, shift)
    (1, 1, 1, 0, 0), (1, 8, 8, 0, 0), (1, 4096, 1000, 0, 0), (1, 700, 4099, 0, 0), (2, 64, 14336, 0, 0),
    (3, 17, 5, 0, 0), (7, 3, 130, 5, 1), (16, 2048, 256, 8, 0), (31, 64, 200, 8, 8), (32, 520, 96, 0, 0),
    (33, 72, 1001, 3, 2), (64, 1024, 640, 0, 0), (65, 136, 65, 0, 0), (127, 129, 131, 0, 0), (128, 256, 128, 0, 0),
    (129, 264, 264, 24, 0), (200, 1000, 1363, 0, 0), (256, 4096, 512, 0, 0), (257, 4096, 64, 0, 0),
    (300, 5, 3, 0, 0), (513, 640, 1, 0, 0), (1000, 1, 700, 0, 0), (1024, 520, 776, 1, 0), (2047, 256, 256, 0, 0),
    (2500, 384, 2056, 64, 8), (4, 4104, 520, 8, 8), (4, 131, 600, 1, 1), (5, 264, 1000, 0, 0),
    (12, 1003, 301, 2, 0), (16, 4100, 3000, 4, 4), (2, 5000, 64, 0, 0),
    (1500, 1800, 2104, 8, 8), (1601, 1803, 2101, 3, 1),
    (600, 200, 1363, 0, 0), (2100, 264, 4097, 0, 1), (150, 256, 217, 24, 0), (401, 768, 5001, 0, 0), (1030, 513, 2044, 0, 4),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_linear_forward(dev, case, dtype):
    M, di, do, gap, shift = SHAPES[case]
    gen = torch.Generator(device=dev).manual_seed(case)
    for k in range(3):
        act = ACTS[(case + 2 * k) % 5]
        bias, res, keep = (case + k) % 2 == 0, k != 1, k != 2
        _, X = rows(gen, M, di, gap, shift, 1.0, dtype, dev)
        _, W = rows(gen, do, di, gap, shift, 1.5 / math.sqrt(di), dtype, dev)
        b = torch.randn(do, generator=gen, device=dev).to(dtype) if bias else None
        _, R = rows(gen, M, do, gap, shift, 1.0, dtype, dev) if res else (None, None)
        yb, Y = rows(gen, M, do, gap, shift, 0, dtype, dev, fill=7.0)
        zb, Z = rows(gen, M, do, gap, shift, 0, dtype, dev, fill=7.0) if keep else (None, None)
        L = tda.LinearDesc(di, do, ACTS.index(act), KIND[dtype])
        ws, wsb = ws_for(tda.TDA_LINEAR_FORWARD, L, M, dev, True)
        tda.tda_linear_forward(L, X, X.stride(0), M, W, W.stride(0), b, R, R.stride(0) if res else 0, Y, Y.stride(0), Z,
                               Z.stride(0) if keep else 0, ws, wsb)
        tda.tda_device_status()
        z = X.to(F64) @ W.to(F64).t()
        S = X.to(F64).abs() @ W.to(F64).abs().t()
        if bias:
            z, S = z + b.to(F64), S + b.to(F64).abs()
        tz = product_bound(di, dtype) * S + 2 * U * S
        y = act64(act, z) + (R.to(F64) if res else 0)
        ty = 1.13 * tz + 2.0 ** -20 * z.abs() + 2 * U * y.abs()
        h = HALF_ULP[dtype]
        fro = 2.4e-3 if dtype == torch.bfloat16 else 1e-6
        close(Y, y, ty + h * (y.abs() + ty) + 1e-38, fro if act == "none" else None)
        beside(yb, M, do, gap, shift, 7.0)
        if keep:
            close(Z, z, tz + h * (z.abs() + tz) + 1e-38, fro)
            beside(zb, M, do, gap, shift, 7.0)


@pytest.mark.parametrize("dtype,gt", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                      (torch.float32, torch.float32)])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_linear_backward(dev, case, dtype, gt):
    M, di, do, gap, shift = SHAPES[case]
    gen = torch.Generator(device=dev).manual_seed(100 + case)
    h, hg = HALF_ULP[dtype], HALF_ULP[gt]
    for k in range(2):
        act = ACTS[(case + 3 * k) % 5]
        beta = [0.0, 1.0, -0.5][(case + k) % 3]
        _, dY = rows(gen, M, do, gap, shift, 0.01, dtype, dev)
        if M > 4:
            dY[1::3] = 0  # padded tokens
        _, Z = rows(gen, M, do, gap, shift, 2.0, dtype, dev)
        _, X = rows(gen, M, di, gap, shift, 1.0, dtype, dev)
        _, W = rows(gen, do, di, gap, shift, 1 / math.sqrt(do), dtype, dev)
        fill = float("nan")
        bb, B = rows(gen, M, do, gap, shift, 0, dtype, dev, fill=7.0) if act != "none" or k else (None, None)
        xb, dX = rows(gen, M, di, gap, shift, 0, dtype, dev, fill=7.0)
        _, dW = rows(gen, do, di, gap, shift, 0.01, gt, dev, fill=None if beta else fill)
        db = torch.randn(do, generator=gen, device=dev).to(gt) if beta else torch.full((do,), fill, dtype=gt, device=dev)
        oldW, oldb = dW.to(F64).clone(), db.to(F64).clone()
        L = tda.LinearDesc(di, do, ACTS.index(act), KIND[dtype])
        ws, wsb = ws_for(tda.TDA_LINEAR_BACKWARD, L, M, dev, True)
        tda.tda_linear_backward(L, dY, dY.stride(0), Z if act != "none" else None, Z.stride(0), M, X, X.stride(0), W,
                                W.stride(0), B, B.stride(0) if B is not None else 0, dX, dX.stride(0), dW,
                                dW.stride(0), db, KIND[gt], beta, ws, wsb)
        tda.tda_device_status()
        b = dY.to(F64) * (slope64(act, Z.to(F64)) if act != "none" else 1)
        tb = 2.0 ** -20 * dY.to(F64).abs() if act != "none" else 0 * b
        hb = h if act != "none" else 0.0  # without an activation the factor is dY, unrounded
        if B is not None:
            close(B, b, tb + h * (b.abs() + tb) + 1e-38)
            beside(bb, M, do, gap, shift, 7.0)
        eb = tb + hb * (b.abs() + tb)  # what the stored factor may be off by
        rnd = (2.4e-3 if act == "none" else 3.5e-3) if dtype == torch.bfloat16 else 1.5e-6
        dx = b @ W.to(F64)
        S = (b.abs() + eb) @ W.to(F64).abs()
        t = product_bound(do, dtype) * S + eb @ W.to(F64).abs()
        close(dX, dx, t + h * (dx.abs() + t) + 1e-38, rnd)
        beside(xb, M, di, gap, shift, 7.0)
        dw = b.t() @ X.to(F64)
        t = product_bound(M, dtype) * ((b.abs() + eb).t() @ X.to(F64).abs()) + eb.t() @ X.to(F64).abs()
        d_b, t_b = b.sum(0), ((M / 8 + 300) * U) * b.abs().sum(0) + tb.sum(0)
        if beta:
            dw, d_b = dw + beta * oldW, d_b + beta * oldb
            t, t_b = t + 2 * U * (oldW.abs() + dw.abs()), t_b + 2 * U * (oldb.abs() + d_b.abs())
        close(dW, dw, t + hg * (dw.abs() + t) + 1e-38, None if beta else rnd)
        close(db, d_b, t_b + hg * (d_b.abs() + t_b) + 1e-38)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_linear_backward_parts(dev, dtype):
    """Each output alone gives what it gives with the others, up to the order of its sums (which may depend on what
    shares the launch); an empty batch scales what is there."""
    M, di, do = 150, 264, 392
    gen = torch.Generator(device=dev).manual_seed(3)
    mk = lambda *s: torch.randn(s, generator=gen, device=dev).to(dtype)
    dY, Z, X, W = mk(M, do), mk(M, do), mk(M, di), mk(do, di)
    L = tda.LinearDesc(di, do, tda.TDA_ACT_SILU, KIND[dtype])
    ws, wsb = ws_for(tda.TDA_LINEAR_BACKWARD, L, M, dev, False)

    def call(want):
        o = dict(B=torch.empty_like(dY), dX=torch.empty_like(X) if "dX" in want else None,
                 dW=torch.empty((do, di), device=dev) if "dW" in want else None,
                 db=torch.empty(do, device=dev) if "db" in want else None)
        tda.tda_linear_backward(L, dY, do, Z, do, M, X if "dW" in want else None, di, W if "dX" in want else None, di,
                                o["B"], do, o["dX"], di, o["dW"], di, o["db"], tda.TDA_F32, 0.0, ws, wsb)
        tda.tda_device_status()
        return o

    full = call(("dX", "dW", "db"))
    Bd = full["B"].to(F64).abs()
    bound = {"dX": 2 * product_bound(do, dtype) * (Bd @ W.to(F64).abs()) + 2 * HALF_ULP[dtype] * full["dX"].to(F64).abs(),
             "dW": 2 * product_bound(M, dtype) * (Bd.t() @ X.to(F64).abs()) + 2 * U * full["dW"].to(F64).abs(),
             "db": 0 * full["db"].to(F64)}
    for want in (("dX",), ("dW",), ("db",), ()):
        o = call(want)
        assert torch.equal(o["B"], full["B"])
        for w in want:
            close(o[w], full[w].to(F64), bound[w])
    # the factor in dY's place
    g = dY.clone()
    dX = torch.empty_like(X)
    tda.tda_linear_backward(L, g, do, Z, do, M, None, 0, W, di, g, do, dX, di, None, 0, None, tda.TDA_F32, 0.0, ws, wsb)
    assert torch.equal(g, full["B"])
    close(dX, full["dX"].to(F64), bound["dX"])
    # no tokens
    dW, db = full["dW"].clone(), full["db"].clone()
    tda.tda_linear_backward(L, None, do, None, do, 0, None, di, None, di, None, do, None, di, dW, di, db, tda.TDA_F32,
                            0.5, None, 0)
    assert torch.equal(dW, 0.5 * full["dW"]) and torch.equal(db, 0.5 * full["db"])
    tda.tda_linear_backward(L, None, do, None, do, 0, None, di, None, di, None, do, None, di, dW, di, None, tda.TDA_F32,
                            0.0, None, 0)
    assert bool((dW == 0).all())
    tda.tda_linear_forward(L, None, di, 0, None, di, None, None, 0, None, do, None, 0, None, 0)


def test_linear_residual_in_place(dev):
    M, di, do = 300, 512, 512
    X = torch.randn(M, di, device=dev).bfloat16()
    W = (torch.randn(do, di, device=dev) / 20).bfloat16()
    R = torch.randn(M, do, device=dev).bfloat16()
    Y = torch.empty_like(R)
    L = tda.LinearDesc(di, do, tda.TDA_ACT_NONE, tda.TDA_BF16)
    tda.tda_linear_forward(L, X, di, M, W, di, None, R, do, Y, do)
    S = R.clone()
    tda.tda_linear_forward(L, X, di, M, W, di, None, S, do, S, do)
    assert torch.equal(S, Y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", ACTS)
def test_activations_over_their_whole_range(dev, act, dtype):
    """W = I: Y = act(x) and B = act'(x) for x from tiny to huge, where formulas overflow or cancel."""
    mags = torch.cat([torch.logspace(-30, 30, 121, dtype=F64), torch.linspace(0, 30, 391, dtype=F64)])
    x = torch.cat([mags, -mags]).to(device=dev).to(dtype).view(16, 64)
    I = torch.eye(64, device=dev).to(dtype)
    L = tda.LinearDesc(64, 64, ACTS.index(act), KIND[dtype])
    Y, Z, B = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    ws, wsb = ws_for(tda.TDA_LINEAR_BACKWARD, L, 16, dev, False)
    tda.tda_linear_forward(L, x, 64, 16, I, 64, None, None, 0, Y, 64, Z, 64, ws, wsb)
    one = torch.ones_like(x)
    tda.tda_linear_backward(L, one, 64, Z, 64, 16, None, 0, None, 0, B, 64, None, 0, None, 0, None, tda.TDA_F32, 0.0, ws,
                            wsb)
    tda.tda_device_status()
    h = HALF_ULP[dtype]
    assert bool(((Z.to(F64) - x.to(F64)).abs() <= 2.0 ** -22 * x.to(F64).abs() + 1e-37).all())
    z = Z.to(F64)
    # a value z (1 - p): error of p times z, and of p itself in its tail: exp of an argument of size a is good to a 2^-23
    big = z.abs().clamp(max=200.0) ** 2
    y = act64(act, z)
    close(Y, y, (8 * U + big * 4 * U) * y.abs() + h * y.abs() * 1.01 + 2.0 ** -21 * x.to(F64).abs().clamp(max=40) * 0.01
          + 2.0 ** -22 * x.to(F64).abs() + 1e-37)
    s = slope64(act, z)
    s = torch.where(torch.isfinite(s), s, (z > 0).to(F64))  # where fp64's own formula overflows
    close(B, s, 2.0 ** -20 + h * s.abs() * 1.01)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "none"])
def test_linear_gradients_against_differences(dev, act):
    """Directional central differences of <G, Y> in X, W and the bias. With step h the quotient is off by at most
    h^2 / 6 times the third derivative (below 2 for these functions) of each output along the direction, and
    by the forward pass's own error over h."""
    M, di, do, h = 24, 40, 56, 2.0 ** -4
    gen = torch.Generator(device=dev).manual_seed(11)
    mk = lambda *s: torch.randn(s, generator=gen, device=dev)
    X, W, b, G = mk(M, di), mk(do, di) / math.sqrt(di), mk(do), mk(M, do)
    L = tda.LinearDesc(di, do, ACTS.index(act), tda.TDA_F32)
    ws, wsb = ws_for(tda.TDA_LINEAR_BACKWARD, L, M, dev, False)

    def forward(X, W, b):
        Y, Z = torch.empty((M, do), device=dev), torch.empty((M, do), device=dev)
        tda.tda_linear_forward(L, X, di, M, W, di, b, None, 0, Y, do, Z, do, ws, wsb)
        return Y.to(F64), Z

    _, Z = forward(X, W, b)
    B, dX, dW, db = torch.empty_like(Z), torch.empty_like(X), torch.empty_like(W), torch.empty_like(b)
    tda.tda_linear_backward(L, G, do, Z, do, M, X, di, W, di, B, do, dX, di, dW, di, db, tda.TDA_F32, 0.0, ws, wsb)
    tda.tda_device_status()
    for which, grad in ((0, dX), (1, dW), (2, db)):
        base = [X, W, b]
        D = mk(*base[which].shape) / math.sqrt(di if which < 2 else 1)
        up, dn = list(base), list(base)
        up[which], dn[which] = base[which] + h * D, base[which] - h * D
        (yu, zu), (yd, zd) = forward(*up), forward(*dn)
        quotient = float((G.to(F64) * (yu - yd)).sum()) / (2 * h)
        dz = ((zu - zd).to(F64) / (2 * h)).abs()
        third = 0.0 if act == "none" else float((G.to(F64).abs() * 2 * dz ** 3).sum()) * h * h / 6
        noise = float(G.to(F64).abs().sum()) * 1e-5 / h
        assert abs(quotient - float((grad.to(F64) * D.to(F64)).sum())) <= third + noise


def test_linear_non_finite_stays_in_its_rows(dev):
    M, di, do = 70, 128, 136
    for dtype in (torch.bfloat16, torch.float32):
        X = torch.randn(M, di, device=dev).to(dtype)
        W = torch.randn(do, di, device=dev).to(dtype)
        X[5, 7], X[40, 0] = float("nan"), float("inf")
        W[9, 3] = float("-inf")
        Y = torch.empty((M, do), dtype=dtype, device=dev)
        L = tda.LinearDesc(di, do, tda.TDA_ACT_NONE, KIND[dtype])
        ws, wsb = ws_for(tda.TDA_LINEAR_FORWARD, L, M, dev, False)
        tda.tda_linear_forward(L, X, di, M, W, di, None, None, 0, Y, do, None, 0, ws, wsb)
        bad = torch.zeros((M, do), dtype=torch.bool, device=dev)
        bad[5] = bad[40] = True
        bad[:, 9] = True
        assert torch.equal(~torch.isfinite(Y), bad)


def test_linear_fp32_range(dev):
    """Values whose lower planes leave bf16's normal range, and values near the largest."""
    M, di, do = 8, 64, 24
    X = torch.randn(M, di, device=dev)
    W = torch.randn(do, di, device=dev)
    L = tda.LinearDesc(di, do, tda.TDA_ACT_NONE, tda.TDA_F32)
    ws, wsb = ws_for(tda.TDA_LINEAR_FORWARD, L, M, dev, False)
    for sx, sw in ((1e-30, 1.0), (1e37, 1e-30), (3e-38, 1e20)):
        x, w = X * sx, W * sw
        Y = torch.empty((M, do), device=dev)
        tda.tda_linear_forward(L, x, di, M, w, di, None, None, 0, Y, do, None, 0, ws, wsb)
        ref = x.to(F64) @ w.to(F64).t()
        S = x.to(F64).abs() @ w.to(F64).abs().t()
        # planes below 2^-133 (bf16's smallest) are lost: an absolute error of 2^-134 per element
        lost = 2.0 ** -133 * (w.to(F64).abs().sum(1)[None] + x.to(F64).abs().sum(1)[:, None])
        close(Y, ref, product_bound(di, torch.float32) * S + lost + U * ref.abs())
    big = torch.full((1, 8), 3.4e38, device=dev)
    w = torch.zeros((8, 8), device=dev)
    w[:, 0] = 1.0
    Y = torch.empty((1, 8), device=dev)
    L = tda.LinearDesc(8, 8, tda.TDA_ACT_NONE, tda.TDA_F32)
    tda.tda_linear_forward(L, big, 8, 1, w, 8, None, None, 0, Y, 8, None, 0, ws, wsb)
    assert float((Y / big - 1).abs().max()) <= 8 * U


def test_linear_reproducible_and_on_a_stream(dev):
    M, di, do = 40, 4096, 1024
    X, W = torch.randn(M, di, device=dev).bfloat16(), torch.randn(do, di, device=dev).bfloat16()
    L = tda.LinearDesc(di, do, tda.TDA_ACT_NONE, tda.TDA_BF16)
    s = torch.cuda.Stream()
    got = []
    s.wait_stream(torch.cuda.current_stream())
    for k in range(4):
        Y = torch.empty((M, do), dtype=torch.bfloat16, device=dev)
        with torch.cuda.stream(s if k % 2 else torch.cuda.current_stream()):
            tda.tda_linear_forward(L, X, di, M, W, di, None, None, 0, Y, do)
        got.append(Y)
    torch.cuda.synchronize()
    assert all(torch.equal(got[0], g) for g in got)


def test_linear_in_a_graph(dev):
    M, di, do = 96, 200, 136
    L = tda.LinearDesc(di, do, tda.TDA_ACT_GELU, tda.TDA_F32)
    X, W, dY = (torch.randn(s, device=dev) for s in ((M, di), (do, di), (M, do)))
    Y, Z, B, dX, dW, db = (torch.empty(s, device=dev) for s in ((M, do), (M, do), (M, do), (M, di), (do, di), (do,)))
    ws, wsb = ws_for(tda.TDA_LINEAR_BACKWARD, L, M, dev, False)

    def step():
        tda.tda_linear_forward(L, X, di, M, W, di, None, None, 0, Y, do, Z, do, ws, wsb)
        tda.tda_linear_backward(L, dY, do, Z, do, M, X, di, W, di, B, do, dX, di, dW, di, db, tda.TDA_F32, 0.0, ws, wsb)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    X.copy_(torch.randn(M, di, device=dev))
    step()
    want = [t.clone() for t in (Y, Z, B, dX, dW, db)]
    for t in (Y, Z, B, dX, dW, db):
        t.fill_(float("nan"))
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, w) for t, w in zip((Y, Z, B, dX, dW, db), want))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_linear_padded_rows_with_non_finite_z(dev, act, dtype):
    """A padded token's pre-activation may hold anything: its factor is zero, and so is its share of dX, dW, db."""
    M, di, do = 90, 136, 200
    mk = lambda *s: torch.randn(s, device=dev).to(dtype)
    dY, Z, X, W = mk(M, do), mk(M, do), mk(M, di), mk(do, di)
    dY[7::9] = 0
    clean = Z.clone()
    Z[7], Z[16], Z[25] = float("nan"), float("inf"), float("-inf")
    L = tda.LinearDesc(di, do, ACTS.index(act), KIND[dtype])
    ws, wsb = ws_for(tda.TDA_LINEAR_BACKWARD, L, M, dev, False)
    got = []
    for z in (Z, clean):
        B, dX, dW, db = torch.empty_like(dY), torch.empty_like(X), torch.empty(do, di, device=dev), torch.empty(do, device=dev)
        tda.tda_linear_backward(L, dY, do, z, do, M, X, di, W, di, B, do, dX, di, dW, di, db, tda.TDA_F32, 0.0, ws, wsb)
        got.append((B, dX, dW, db))
    assert bool((got[0][0][7::9] == 0).all())
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_linear_offsets_past_32_bits(dev):
    """Tall views in wide rows: elements more than 2^31 from the tensors' starts, both passes."""
    M, di, do, ld = 270_000, 64, 40, 8192
    gen = torch.Generator(device=dev).manual_seed(1)
    wide = lambda n: torch.empty((M, ld), dtype=torch.bfloat16, device=dev)[:, :n]
    X, Y, dX = wide(di), wide(do), wide(di)
    X.copy_(torch.randn((M, di), generator=gen, device=dev))
    W = (torch.randn((do, di), generator=gen, device=dev) / 8).bfloat16()
    L = tda.LinearDesc(di, do, tda.TDA_ACT_NONE, tda.TDA_BF16)
    tda.tda_linear_forward(L, X, ld, M, W, di, None, None, 0, Y, ld)
    tda.tda_device_status()
    ref = X.to(F64) @ W.to(F64).t()
    close(Y, ref, product_bound(di, torch.bfloat16) * (X.to(F64).abs() @ W.to(F64).abs().t()) + 1.01 * 2.0 ** -8 * ref.abs()
          + 1e-4, 2.4e-3)
    ws, wsb = ws_for(tda.TDA_LINEAR_BACKWARD, L, M, dev, False)
    tda.tda_linear_backward(L, Y, ld, None, 0, M, None, 0, W, di, None, 0, dX, ld, None, 0, None, tda.TDA_F32, 0.0, ws, wsb)
    tda.tda_device_status()
    ref = Y.to(F64) @ W.to(F64)
    close(dX, ref, product_bound(do, torch.bfloat16) * (Y.to(F64).abs() @ W.to(F64).abs()) + 1.01 * 2.0 ** -8 * ref.abs()
          + 1e-4, 2.4e-3)
