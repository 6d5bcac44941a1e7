"""Embedding lookup, its gradient and gradient clipping against plain fp64 implementations, at the sizes, ids,
strides and values where they can go wrong. Tolerances come from the arithmetic: u = 2^-24 per fp32 operation on
the sum of magnitudes, half an ulp of the output type for the one rounding at the end."""
import numpy as np
import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # unit roundoff 2^-p, p = 24 and 8 bits
KIND = {torch.float32: tda.TDA_F32, torch.bfloat16: tda.TDA_BF16}
INDEX = {torch.int32: tda.TDA_I32, torch.int64: tda.TDA_I64}


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


def wide(rows, cols, gap, shift, dtype, dev, gen, fill=None):
    """rows x cols in rows of cols + gap, the first value `shift` values into its buffer."""
    buf = torch.empty(rows * (cols + gap) + shift + 16, dtype=torch.float32, device=dev)
    buf = (buf.normal_(generator=gen) if fill is None else buf.fill_(fill)).to(dtype)
    return buf, buf[shift:shift + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]


# ------------------------------------------------------------------ lookup
LOOKUPS = [
    # (n, V, d, gap, shift, scale)
    (1, 1, 1, 0, 0, 1.0), (1, 7, 8, 0, 0, 2.0), (3, 50, 4096, 0, 0, 1.0), (37, 1000, 1363, 0, 0, 0.25),
    (129, 333, 72, 8, 8, 1.0), (64, 100, 1030, 2, 2, 3.0), (1000, 5, 33, 31, 1, 1.0), (5, 9, 14336, 0, 0, 64.0),
    (257, 4000, 130, 6, 4, 1.0),
]


@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", LOOKUPS)
def test_embedding_forward(dev, case, dtype, index):
    n, V, d, gap, shift, scale = case
    gen = torch.Generator(device=dev).manual_seed(n * 7 + d)
    _, E = wide(V, d, gap, shift, dtype, dev, gen)
    tok = torch.randint(0, V, (n,), generator=gen, device=dev)
    if n > 4:  # padding, and ids outside the table
        tok[1], tok[2], tok[n - 1] = -1, V, V + 12345
        tok[3] = torch.iinfo(index).min
    tok = tok.to(index)
    buf, out = wide(n, d, gap, shift, dtype, dev, gen, fill=7.0)
    tda.tda_embedding_forward(KIND[dtype], E, E.stride(0), V, d, INDEX[index], tok, n, scale, out, out.stride(0))
    tda.tda_device_status()
    t = tok.cpu().long()
    ref = torch.zeros((n, d), dtype=torch.float64)
    for i in range(n):
        if t[i] >= V:
            ref[i] = float("nan")
        elif t[i] >= 0:
            ref[i] = scale * E[t[i]].double().cpu()
    # one fp32 product and one rounding: the correctly rounded result itself
    assert torch.equal(torch.nan_to_num(out.cpu(), nan=99.0), torch.nan_to_num(ref.to(torch.float32).to(dtype), nan=99.0))
    inside = torch.zeros(buf.numel(), dtype=torch.bool)
    inside[shift:shift + n * (d + gap)].view(n, d + gap)[:, :d] = True
    assert (buf.cpu()[~inside] == 7.0).all()  # nothing beside the rows


def test_embedding_forward_long_table(dev):
    """Offsets past 2^31 elements: the last rows of a table of 2.2e9 values."""
    V, d = 550_000, 4096
    E = torch.empty((V, d), dtype=torch.bfloat16, device=dev)
    E[-2:] = torch.arange(2 * d, device=dev).view(2, d).to(torch.bfloat16)
    E[0] = 1.0
    tok = torch.tensor([V - 1, 0, V - 2], device=dev)
    out = torch.empty((3, d), dtype=torch.bfloat16, device=dev)
    tda.tda_embedding_forward(tda.TDA_BF16, E, d, V, d, tda.TDA_I64, tok, 3, 1.0, out, d)
    assert torch.equal(out, E[tok])


# ------------------------------------------------------------------ gradient
def run_grad(dout, V, tok, scale, gt, dE, beta):
    n, d = dout.shape
    wsb = tda.tda_embedding_workspace_size(V, d, n)
    ws = torch.full((max(wsb, 1),), 0x7F, dtype=torch.uint8, device=dE.device)  # NaN-like garbage
    tda.tda_embedding_backward(KIND[dout.dtype], dout, dout.stride(0), V, d, INDEX[tok.dtype], tok, n, scale, KIND[gt],
                               dE, dE.stride(0), beta, ws, wsb)
    tda.tda_device_status()


def check_grad(dout, V, tok, scale, gt, got, beta, old):
    t = tok.long()
    live = (t >= 0) & (t < V)
    x = dout.double()[live]
    ref = beta * old.double() if beta else torch.zeros(old.shape, dtype=torch.float64, device=old.device)
    ref = ref.index_add(0, t[live], scale * x)
    size = torch.zeros(old.shape, dtype=torch.float64, device=old.device).index_add(0, t[live], abs(scale) * x.abs())
    if beta:
        size += abs(beta) * old.double().abs()
    count = torch.zeros(V, dtype=torch.float64, device=old.device).index_add(
        0, t[live], torch.ones(int(live.sum()), dtype=torch.float64, device=old.device)).unsqueeze(1)
    tol = (count + 3) * U * size + HALF_ULP[gt] * (ref.abs() + (count + 3) * U * size) + 1e-40
    err = (got.double() - ref).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    if beta == 0:
        untouched = count.squeeze(1) == 0
        assert bool((got[untouched] == 0).all())


GRADS = [
    # (n, V, d, gap, shift, kind of ids)
    (0, 5, 16, 0, 0, "uniform"), (1, 1, 1, 0, 0, "uniform"), (1, 300, 4096, 0, 0, "uniform"),
    (31, 40, 64, 0, 0, "uniform"), (32, 3, 1363, 0, 0, "uniform"), (33, 1000, 72, 8, 8, "zipf"),
    (64, 64, 130, 2, 2, "same"), (65, 9, 24, 0, 0, "same"), (1000, 33, 200, 0, 0, "zipf"),
    (4096, 32000, 256, 0, 0, "zipf"), (8192, 100, 96, 0, 0, "uniform"), (8191, 131072, 40, 0, 0, "last"),
    (8193, 50021, 40, 0, 0, "zipf"), (20000, 511, 48, 0, 0, "uniform"), (20000, 512, 17, 3, 1, "zipf"),
    (40000, 262144, 32, 0, 0, "zipf"), (100000, 7, 16, 0, 0, "same"), (150000, 70000, 8, 0, 0, "zipf"),
    (300000, 1 << 20, 8, 0, 0, "zipf"), (5000, 100, 64, 0, 0, "padding"), (9000, 100, 64, 0, 0, "padding"),
]


@pytest.mark.parametrize("types", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16),
                                   (torch.float32, torch.float32)])
@pytest.mark.parametrize("case", GRADS)
def test_embedding_backward(dev, case, types):
    n, V, d, gap, shift, ids = case
    ti, gt = types
    gen = torch.Generator(device=dev).manual_seed(n + 3 * V + d)
    _, dout = wide(n, d, gap, shift, ti, dev, gen)
    u = torch.rand((n,), generator=gen, device=dev, dtype=torch.float64)
    if ids == "uniform":
        tok = (u * V).long()
    elif ids == "zipf":
        tok = (torch.exp(u * np.log(V + 1.0)).long() - 1).clamp(0, V - 1)
    elif ids == "same":
        tok = torch.full((n,), V - 1, device=dev)
    elif ids == "last":
        tok = torch.full((n,), V - 1, device=dev)
        tok[: n // 2] = 0
    else:
        tok = torch.full((n,), -1, device=dev)
    if ids in ("zipf", "uniform") and n > 10:  # padding and ids outside the table count for nothing
        tok[3::17] = -1
        tok[5::41] = V
        tok[6::101] = 2 ** 31 - 1
    tok = tok.to(torch.int32 if n % 2 else torch.int64)
    for beta in (0.0, 1.0, -0.5):
        _, dE = wide(V, d, gap, shift, gt, dev, gen)
        old = dE.clone()
        if beta == 0.0:
            dE.fill_(float("nan"))
        run_grad(dout, V, tok, 1.5, gt, dE, beta)
        check_grad(dout, V, tok, 1.5, gt, dE, beta, old)


def test_embedding_backward_is_reproducible(dev):
    gen = torch.Generator(device=dev).manual_seed(5)
    for n, V in ((6000, 500), (50000, 3000)):
        dout = torch.randn((n, 64), generator=gen, device=dev)
        tok = (torch.rand((n,), generator=gen, device=dev) ** 4 * V).int()
        got = []
        for _ in range(3):
            dE = torch.empty((V, 64), device=dev)
            run_grad(dout, V, tok, 1.0, torch.float32, dE, 0.0)
            got.append(dE)
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_embedding_gradient_is_the_lookups(dev):
    """Central differences of <G, lookup(E)> in every entry of a small table, in fp64 from fp32 outputs whose
    inputs are multiples of 2^-6 (all sums exact)."""
    V, d, n = 6, 5, 11
    gen = torch.Generator(device=dev).manual_seed(2)
    E = torch.randint(-64, 64, (V, d), generator=gen, device=dev).float() / 64
    G = torch.randint(-64, 64, (n, d), generator=gen, device=dev).float() / 64
    tok = torch.tensor([0, 3, 3, -1, 5, 0, 3, 1, 1, 3, 5], device=dev)
    dE = torch.empty_like(E)
    run_grad(G, V, tok, 2.0, torch.float32, dE, 0.0)

    def loss(e):
        out = torch.empty((n, d), device=dev)
        tda.tda_embedding_forward(tda.TDA_F32, e, d, V, d, tda.TDA_I64, tok, n, 2.0, out, d)
        return float((out.double() * G.double()).sum())

    h = 0.5
    for v in range(V):
        for c in range(d):
            step = torch.zeros_like(E)
            step[v, c] = h
            assert float(dE[v, c]) == (loss(E + step) - loss(E - step)) / (2 * h)


def test_embedding_on_another_stream(dev):
    s = torch.cuda.Stream()
    n, V, d = 3000, 200, 64
    tok = torch.randint(0, V, (n,), device=dev)
    dout = torch.randn((n, d), device=dev)
    dE = torch.empty((V, d), device=dev)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run_grad(dout, V, tok, 1.0, torch.float32, dE, 0.0)
    torch.cuda.current_stream().wait_stream(s)
    check_grad(dout, V, tok, 1.0, torch.float32, dE, 0.0, torch.zeros_like(dE))


# ------------------------------------------------------------------ norm and clipping
def clip(tensors, max_norm, outs=None, dev="cuda"):
    refs = tda.tensor_list(tensors, outs)
    wsb = tda.tda_grad_clip_workspace_size(refs, len(tensors))
    ws = torch.full((wsb,), 0x7F, dtype=torch.uint8, device=dev)
    norm = torch.full((1,), 7.0, device=dev)
    tda.tda_grad_clip(refs, len(tensors), max_norm, norm, ws, wsb)
    tda.tda_device_status()
    return norm


def ref_norm(tensors):
    return float(torch.sqrt(sum((t.double() ** 2).sum() for t in tensors))) if tensors else 0.0


SIZES = [[1], [0], [], [3, 0, 5], [8192], [8191, 8193], [255, 256, 257, 4096, 12], [1000003], [40000] * 3 + [17],
         [5] * 1100, [2_000_000, 1, 3_000_000]]


@pytest.mark.parametrize("max_norm", [0.5, 1e6, float("inf")])
@pytest.mark.parametrize("dtypes", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s, default=0)}")
def test_grad_clip(dev, sizes, dtypes, max_norm):
    gen = torch.Generator(device=dev).manual_seed(len(sizes) + sum(sizes))
    kinds = {"f32": [torch.float32], "bf16": [torch.bfloat16], "mixed": [torch.float32, torch.bfloat16]}[dtypes]
    # every third tensor starts one element past a 16-byte boundary
    ts = [torch.randn(n + 1, generator=gen, device=dev).to(kinds[i % len(kinds)])[1 if i % 3 == 2 else 0:][:n]
          for i, n in enumerate(sizes)]
    want = ref_norm(ts)
    outs = [torch.full((t.numel() + 8,), 9.0, dtype=t.dtype, device=dev)[:t.numel()] for t in ts]
    norm = clip(ts, max_norm, outs, dev)
    assert abs(float(norm) - want) <= 20 * U * want
    c = 1.0 if want <= max_norm else max_norm / want
    for t, o in zip(ts, outs):
        tol = (23 * U + HALF_ULP[t.dtype] * 1.0001) * (c * t.double()).abs()
        assert bool(((o.double() - c * t.double()).abs() <= tol).all())
    # in place: the same values
    norm2 = clip(ts, max_norm, None, dev)
    assert torch.equal(norm, norm2)
    for t, o in zip(ts, outs):
        assert torch.equal(t, o)


def test_grad_clip_leaves_neighbours_and_skips_none(dev):
    buf = torch.ones(4096, device=dev)
    a, b = buf[10:1000], buf[1001:3000]
    oa = torch.full((2000,), 5.0, device=dev)
    norm = clip([a, b], 1.0, [oa[3:993], None], dev)
    want = np.sqrt(990 + 1999)
    assert abs(float(norm) - want) <= 20 * U * want
    assert (buf == 1).all() and (oa[:3] == 5).all() and (oa[993:] == 5).all()
    assert float((oa[3:993].double() - 1 / want).abs().max()) <= 25 * U / want


@pytest.mark.parametrize("value", [3e38, 1e30, 1e-30, 1e-38, 1e-44, 0.0])
@pytest.mark.parametrize("n", [1, 5000, 20000])
def test_grad_clip_whole_range(dev, value, n):
    """Squares that overflow or vanish in fp32: the norm is right as long as it is an fp32 number."""
    t = torch.full((n,), value / np.sqrt(n) if value > 1e20 else value, device=dev)
    x = float(t[0].double())
    want = x * np.sqrt(n)
    norm = clip([t], float("inf"), None, dev)
    assert abs(float(norm) - want) <= 20 * U * want + 1.5e-45


def test_grad_clip_non_finite(dev):
    for bad in (float("inf"), float("nan")):
        t = torch.ones(10000, device=dev)
        t[1234] = bad
        u = torch.ones(7, device=dev, dtype=torch.bfloat16)
        ot, ou = torch.zeros_like(t), torch.zeros_like(u)
        norm = float(clip([t, u], 1.0, [ot, ou], dev))
        if np.isnan(bad):
            assert np.isnan(norm) and bool(ot.isnan().all()) and bool(ou.isnan().all())
        else:
            assert np.isinf(norm) and bool((ou == 0).all()) and bool(ot[1234].isnan()) and float(ot[0]) == 0


def test_train_ops_capture_in_a_graph(dev):
    n, V, d = 700, 90, 64
    tok = torch.randint(0, V, (n,), device=dev)
    E = torch.randn((V, d), device=dev)
    out, dE = torch.empty((n, d), device=dev), torch.empty((V, d), device=dev)
    clipped, norm = torch.empty_like(dE), torch.empty(1, device=dev)
    wsb = tda.tda_embedding_workspace_size(V, d, n)
    refs = tda.tensor_list([dE], [clipped])
    cwb = tda.tda_grad_clip_workspace_size(refs, 1)
    ws, cws = torch.empty(wsb, dtype=torch.uint8, device=dev), torch.empty(cwb, dtype=torch.uint8, device=dev)

    def step():
        tda.tda_embedding_forward(tda.TDA_F32, E, d, V, d, tda.TDA_I64, tok, n, 1.0, out, d)
        tda.tda_embedding_backward(tda.TDA_F32, out, d, V, d, tda.TDA_I64, tok, n, 1.0, tda.TDA_F32, dE, d, 0.0, ws, wsb)
        tda.tda_grad_clip(refs, 1, 1.0, norm, cws, cwb)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    E.copy_(torch.randn((V, d), device=dev))
    tok.copy_(torch.randint(0, V, (n,), device=dev))
    step()
    want = [x.clone() for x in (out, dE, clipped, norm)]
    for x in (out, dE, clipped, norm):
        x.fill_(float("nan"))
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for x, w in zip((out, dE, clipped, norm), want))


def test_grad_clip_many_tables(dev):
    """More tensors than one launch holds, empty ones among them, some left unclipped."""
    gen = torch.Generator(device=dev).manual_seed(9)
    ts = [torch.randn(0 if i % 7 == 3 else 1 + 37 * (i % 50), generator=gen, device=dev) for i in range(900)]
    outs = [None if i % 11 == 5 else torch.full_like(t, 9.0) for i, t in enumerate(ts)]
    want = ref_norm(ts)
    norm = clip(ts, 2.0, outs, dev)
    assert abs(float(norm) - want) <= 20 * U * want
    c = 2.0 / want
    for t, o in zip(ts, outs):
        if o is not None:
            assert bool(((o.double() - c * t.double()).abs() <= 24 * U * (c * t.double()).abs()).all())


def test_embedding_backward_long_table(dev):
    """Gradient rows more than 2^31 elements from the table's start, short and long lists of tokens."""
    V, d = 540_000, 4096
    dE = torch.empty((V, d), dtype=torch.bfloat16, device=dev)
    gen = torch.Generator(device=dev).manual_seed(4)
    for n in (600, 9000):
        tok = torch.randint(V - 50, V, (n,), generator=gen, device=dev)
        dout = torch.randn((n, d), generator=gen, device=dev).bfloat16()
        dE.fill_(3.0)
        run_grad(dout, V, tok, 1.0, torch.bfloat16, dE, 0.0)
        assert bool((dE[: V - 50] == 0).all())
        check_grad(dout, 50, tok - (V - 50), 1.0, torch.bfloat16, dE[V - 50:], 0.0, torch.zeros((50, d), device=dev))
