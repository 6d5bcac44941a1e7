"""Attention and its backward pass against the definition in 64 bits, at the lengths, masks, strides and values where
they can go wrong. The bounds are attention_reference.Bounds'."""
import math

import pytest
import torch

import paper_2609_38767_gb300 as tda
from attention_reference import Bounds, attention, bias_of, by_bucket, gradients, seen_by
from paper_2609_38767_gb300 import build as tbuild

pytestmark = pytest.mark.gpu

KIND = {torch.float32: tda.TDA_F32, torch.bfloat16: tda.TDA_BF16}
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


def wide(rows, cols, gap, shift, dtype, dev, gen, fill=None, sigma=1.0):
    """rows x cols in rows of cols + gap, the first value `shift` values into its buffer."""
    buf = torch.empty(rows * (cols + gap) + shift + 16, dtype=torch.float32, device=dev)
    buf = (buf.normal_(0, sigma, generator=gen) if fill is None else buf.fill_(fill)).to(dtype)
    return buf, buf[shift:shift + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]


def ranges_for(kind, N, T, gen, dev):
    """Ranges of a kind; None for the plain masks."""
    if kind in ("causal", "full"):
        return None
    at = torch.arange(T).expand(N, T)
    g = torch.Generator().manual_seed(T)
    if kind == "causal_range":
        return torch.stack([torch.zeros_like(at), at + 1], 2).int().to(dev)
    if kind == "window":
        return torch.stack([at - 70, at + 1], 2).int().to(dev)  # negative starts are clamped
    if kind == "any":  # nothing, one key, everything, the far end, past the end
        lo, n = torch.randint(-3, T, (N, T), generator=g), torch.randint(0, T + 5, (N, T), generator=g)
        n[torch.rand((N, T), generator=g) < 0.2] = 0
        n[torch.rand((N, T), generator=g) < 0.1] = 1
        return torch.stack([lo, lo + n], 2).int().to(dev)
    if kind == "docs":
        doc = (torch.rand((N, T), generator=g) < 3.5 / max(T, 4)).long().cumsum(1)
        doc[torch.rand((N, T), generator=g) < 0.03] = -1
        doc[:, T - T // 7:] = -1
        pre = (torch.rand((N, T), generator=g) < 0.9).int().to(dev)
        out = torch.empty((N, T, 2), dtype=torch.int32, device=dev)
        tda.tda_attention_ranges(N, T, doc.int().to(dev), pre, True, 0, out)
        return out
    if kind == "none":
        return torch.zeros((N, T, 2), dtype=torch.int32, device=dev)
    raise KeyError(kind)


class Problem:
    def __init__(self, dev, N, T, H, KV, hd, dtype, mask, cap=0.0, buckets=0, reach=0, slope=False, layout="packed", seed=0,
                 sigma=1.0, garbage=True):
        self.gen = gen = torch.Generator(device=dev).manual_seed(1000 * T + 10 * H + hd + seed)
        self.N, self.T, self.H, self.KV, self.hd, self.dtype, self.dev = N, T, H, KV, hd, dtype, dev
        self.scale, self.cap, self.reach, self.buckets = 1.0 / math.sqrt(hd), cap, reach, buckets
        M, a, b = N * T, H * hd, KV * hd
        if layout == "packed":
            self.buf, x = wide(M, a + 2 * b, 0, 0, dtype, dev, gen, sigma=sigma)
            self.Q, self.K, self.V = x[:, :a], x[:, a:a + b], x[:, a + b:]
        else:
            gap, shift = layout
            self.Q, self.K, self.V = (wide(M, c, gap, shift, dtype, dev, gen, sigma=sigma)[1] for c in (a, b, b))
        self.range = ranges_for(mask, N, T, gen, dev)
        self.seen = seen_by(self.range, T, N, mask == "causal", dev)
        gap, shift = (0, 0) if layout == "packed" else layout
        self.dO = wide(M, a, gap, shift, dtype, dev, gen)[1]
        if garbage and self.range is not None:
            dead = ~self.seen.any(1).reshape(-1)
            idle = ~self.seen.any(2).reshape(-1)
            self.K[dead], self.V[dead], self.Q[idle], self.dO[idle] = math.nan, math.inf, math.nan, math.nan
        self.bucket = self.table = self.slope = None
        if buckets:
            self.bucket = torch.randint(-1, buckets, (2 * reach + 1,), generator=gen, device=dev).int()
            self.table = torch.randn((buckets, H), generator=gen, device=dev).to(dtype)
        if slope:
            self.slope = torch.rand(H, generator=gen, device=dev) * 0.1
        self.bias = bias_of(T, H, self.bucket, reach, self.table, self.slope, dev) if buckets or slope else None
        self.L = tda.AttentionDesc(N, T, H, KV, hd, KIND[dtype], self.scale, cap, mask == "causal", buckets, reach)
        self.gap, self.shift = gap, shift

    def heads(self, x, n):
        return x.reshape(self.N, self.T, n, self.hd).transpose(1, 2)

    def exact(self):
        return attention(self.heads(self.Q, self.H), self.heads(self.K, self.KV), self.heads(self.V, self.KV), self.seen, self.scale,
                         self.cap, self.bias)

    def forward(self, stream=None):
        M, a = self.N * self.T, self.H * self.hd
        obuf, self.O = wide(M, a, self.gap, self.shift, self.dtype, self.dev, self.gen, fill=7.0)
        self.lse = torch.full((self.N, self.H, self.T), 7.0, device=self.dev)
        wsb = tda.tda_attention_workspace_size(tda.TDA_ATTENTION_FORWARD, self.L)
        ws = torch.full((max(wsb, 1),), 255, dtype=torch.uint8, device=self.dev)
        tda.tda_attention_forward(self.L, self.Q, self.Q.stride(0), self.K, self.K.stride(0), self.V, self.V.stride(0), self.range,
                                  self.bucket, self.table, self.slope, self.O, self.O.stride(0), self.lse, ws, wsb, stream)
        return obuf

    def backward(self, beta=0.0, grad=None, stream=None):
        M, a, b = self.N * self.T, self.H * self.hd, self.KV * self.hd
        made = [wide(M, c, self.gap, self.shift, self.dtype, self.dev, self.gen, fill=7.0) for c in (a, b, b)]
        self.dQ, self.dK, self.dV = (x for _, x in made)
        grad = grad or self.dtype
        self.dtable = torch.full((self.buckets, self.H), 0.5, dtype=grad, device=self.dev) if self.buckets else None
        wsb = tda.tda_attention_workspace_size(tda.TDA_ATTENTION_BACKWARD, self.L)
        ws = torch.full((max(wsb, 1),), 255, dtype=torch.uint8, device=self.dev)
        tda.tda_attention_backward(self.L, self.Q, self.Q.stride(0), self.K, self.K.stride(0), self.V, self.V.stride(0), self.range,
                                   self.bucket, self.table, self.slope, self.O, self.O.stride(0), self.lse, self.dO,
                                   self.dO.stride(0), self.dQ, self.dQ.stride(0), self.dK, self.dK.stride(0), self.dV,
                                   self.dV.stride(0), self.dtable, KIND[grad], beta, ws, wsb, stream)
        return [x for x, _ in made]


def near(got, want, tol, what):
    got = got.double()
    fine = torch.isfinite(want)
    bad = int((~torch.isfinite(got[fine])).sum())
    assert not bad, f"{what}: {bad} of {want.numel()} values not finite"
    same = torch.equal(got[~fine], want[~fine])
    assert same, f"{what}: infinities"
    off = (got - want)[fine].abs() / tol.expand_as(want)[fine]
    most = float(off.max()) if off.numel() else 0.0
    assert most <= 1.0, f"{what}: {most:.3g} of the bound, {int((off > 1).sum())} of {off.numel()} values"


def untouched(buf, p, cols):
    """What lies outside the rows of a wide() tensor still holds its filling."""
    rows = p.N * p.T
    assert (buf[:p.shift] == 7).all() and (buf[p.shift + rows * (cols + p.gap):] == 7).all()
    assert (buf[p.shift:p.shift + rows * (cols + p.gap)].view(rows, cols + p.gap)[:, cols:] == 7).all()


def check_forward(p):
    buf = p.forward()
    tda.tda_device_status()
    f = p.exact()
    bias = p.bias if p.bias is None else p.bias.nan_to_num(neginf=0.0)  # a hidden pair has no weight and no error
    b = Bounds(f, p.dtype, p.T, p.hd, p.cap, bias)
    near(p.heads(p.O, p.H), f["o"], b.o(), "O")
    near(p.lse, f["lse"], b.lse(), "lse")
    untouched(buf, p, p.H * p.hd)
    return f, b


def check_backward(p, f, b, beta=0.0, grad=None, summed=False):
    bufs = p.backward(beta, grad)
    tda.tda_device_status()
    r = gradients(f, p.heads(p.dO, p.H), p.scale, p.KV, p.bucket, p.reach, p.buckets)
    if p.buckets:
        r["dtable"] = r["dtable"] + beta * 0.5
    tol = b.grads(r, p.scale, p.KV, p.bucket, p.reach, p.buckets, {BF: 2.0 ** -8, F32: 2.0 ** -24}[grad or p.dtype], summed)
    near(p.heads(p.dQ, p.H), r["dQ"], tol["dQ"], "dQ")
    near(p.heads(p.dK, p.KV), r["dK"], tol["dK"], "dK")
    near(p.heads(p.dV, p.KV), r["dV"], tol["dV"], "dV")
    if p.buckets:
        near(p.dtable, r["dtable"], tol["dtable"], "dtable")
    for x, c in zip(bufs, (p.H, p.KV, p.KV)):
        untouched(x, p, c * p.hd)


MASKS = ["causal", "full", "window", "any", "docs", "none"]
SHAPES = [
    # (N, T, H, KV, hd)
    (1, 1, 1, 1, 64), (2, 2, 2, 1, 128), (1, 37, 4, 2, 64), (2, 64, 2, 2, 128), (1, 127, 3, 1, 96), (3, 128, 2, 1, 64),
    (1, 129, 2, 2, 128), (1, 255, 4, 1, 80), (2, 257, 2, 2, 128), (1, 300, 2, 1, 8), (1, 513, 2, 1, 64),
    (30, 140, 16, 2, 64), (9, 600, 16, 4, 128),  # more tiles than SMs
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("shape", SHAPES)
def test_attention(dev, shape, mask, dtype):
    p = Problem(dev, *shape, dtype, mask)
    f, b = check_forward(p)
    check_backward(p, f, b)


RICH = [
    # (shape, mask, cap, buckets, reach, slope)
    ((1, 1, 1, 1, 64), "causal", 5.0, 4, 0, True), ((2, 67, 4, 2, 64), "docs", 3.0, 8, 20, False),
    ((1, 200, 2, 1, 128), "causal", 0.0, 32, 128, False), ((2, 200, 2, 2, 64), "full", 0.0, 0, 0, True),
    ((1, 385, 4, 2, 128), "any", 30.0, 40, 300, True), ((1, 640, 2, 1, 64), "causal", 50.0, 32, 128, False),
    ((1, 640, 2, 2, 72), "docs", 0.0, 16, 1000, False), ((3, 130, 2, 1, 128), "full", 20.0, 3, 5, False),
    ((1, 333, 1, 1, 64), "window", 0.0, 300, 150, True),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape,mask,cap,buckets,reach,slope", RICH)
def test_caps_and_biases(dev, shape, mask, cap, buckets, reach, slope, dtype):
    p = Problem(dev, *shape, dtype, mask, cap, buckets, reach, slope, sigma=2.0)
    f, b = check_forward(p)
    check_backward(p, f, b, beta=1.0 if buckets else 0.0)
    if buckets and dtype == BF:
        check_backward(p, f, b, beta=-0.5, grad=F32)


@pytest.mark.parametrize("layout", [(8, 8), (3, 1), (0, 2), (24, 0)])
@pytest.mark.parametrize("dtype,hd", [(BF, 64), (BF, 36), (BF, 33), (F32, 33), (F32, 128)])
def test_strides_and_widths(dev, layout, dtype, hd):
    p = Problem(dev, 2, 150, 4, 2, hd, dtype, "docs", layout=layout)
    f, b = check_forward(p)
    check_backward(p, f, b)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_hidden_by_bias(dev, dtype):
    """Biases of -inf hide pairs, rows of them see nothing; the type's lowest value does not."""
    p = Problem(dev, 1, 140, 2, 1, 64, dtype, "causal", 0.0, 3, 139)
    at = torch.arange(-139, 140, device=dev)
    p.bucket = torch.where(at % 3 == 0, 0, torch.where(at % 3 == 1, 1, 2)).int()
    p.table = torch.tensor([[-math.inf, torch.finfo(dtype).min], [0.5, 0.0], [-math.inf, torch.finfo(dtype).min]], device=dev).to(dtype)
    p.bias = bias_of(140, 2, p.bucket, 139, p.table, None, dev)
    p.forward()
    tda.tda_device_status()
    f = p.exact()
    assert p.lse[0, 0, 0] == -math.inf and (p.O[0, :64] == 0).all()  # the first token's only key is hidden
    b = Bounds(f, dtype, 140, 64, 0.0, torch.zeros((), dtype=torch.float64, device=dev))
    near(p.heads(p.O, 2), f["o"], b.o(), "O")
    p.backward()
    tda.tda_device_status()
    r = gradients(f, p.heads(p.dO, 2), p.scale, 1)
    tol = b.grads(r, p.scale, 1)
    for name in ("dQ", "dK", "dV"):
        near(p.heads(getattr(p, name), 2 if name == "dQ" else 1), r[name], tol[name], name)


def test_equal_calls_give_equal_bits(dev):
    for dtype in (BF, F32):
        p = Problem(dev, 2, 700, 8, 2, 64, dtype, "docs", 30.0, 32, 128)
        got = []
        for _ in range(3):
            p.forward()
            p.backward()
            got.append([x.clone() for x in (p.O, p.lse, p.dQ, p.dK, p.dV, p.dtable)])
        tda.tda_device_status()
        for other in got[1:]:
            assert all(torch.equal(x, y) for x, y in zip(got[0], other))


@pytest.mark.parametrize("buckets", [0, 5])
@pytest.mark.parametrize("cap", [4.0, 30.0, 60.0, 62.3, 62.4, 80.0])
def test_scores_at_the_cap(dev, cap, buckets):
    """Scores that rise and fall from one end of the capped range to the other, within a tile and from tile to tile, and rows
    that stay at the lower end."""
    T, hd = 700, 64
    p = Problem(dev, 1, T, 4, 1, hd, BF, "full", cap, buckets, 40 if buckets else 0, sigma=0.5)
    at = torch.arange(T, device=dev)
    along = torch.stack([torch.sin(at / 40.0) * 3, at / T * 6 - 3, 3 - at / T * 6, (at // 128 % 2) * 6.0 - 3])  # of the keys, by head
    if buckets:
        p.table[1] = -math.inf
        p.table[2] = 4.0
        p.bias = bias_of(T, 4, p.bucket, 40, p.table, None, dev)
    p.Q[:, :] = 0
    p.K[:, :] = 0
    for h in range(4):  # a direction of its own for each head's queries, of either sign and some weak
        p.Q[:, h * hd + h] = torch.where(at % 3 == 0, 1.0, torch.where(at % 3 == 1, -1.0, 0.05)).to(BF)
        p.K[:, h] = (along[h] * cap / p.scale).to(BF)
    p.Q[:, 8], p.Q[:, hd + 8] = 1.0, -1.0
    p.K[:, 8] = -(cap / p.scale)
    f, b = check_forward(p)
    check_backward(p, f, b, beta=0.5 if buckets else 0.0, grad=F32)


@pytest.mark.parametrize("mask", ["causal", "docs", "any"])
@pytest.mark.parametrize("T,hd", [(2, 64), (6, 96), (17, 128), (40, 64), (100, 80), (128, 128)])
def test_gradients_of_few_keys(dev, T, hd, mask):
    """Keys of one tile: the gradients do without the stored O and the errors that its rounding has left in it."""
    p = Problem(dev, 3, T, 4, 2, hd, BF, mask, 0.0 if T % 4 else 30.0, 7, 9, sigma=1.3)
    f, b = check_forward(p)
    check_backward(p, f, b, grad=F32, summed=True)


def test_gradients_of_narrow_windows(dev):
    """The same for four keys a row in long examples, but where they lie in two tiles."""
    T = 300
    p = Problem(dev, 2, T, 4, 2, 64, BF, "full", 0.0, 5, 9, sigma=1.3)
    at = torch.arange(T, device=dev)
    p.range = torch.stack([(at - 3).clamp(min=0), at + 1], 1).int().expand(2, T, 2).contiguous()
    p.seen = (at >= p.range[..., :1]) & (at < p.range[..., 1:])
    f, b = check_forward(p)
    p.backward(grad=F32)
    tda.tda_device_status()
    r = gradients(f, p.heads(p.dO, 4), p.scale, 2, p.bucket, p.reach, p.buckets)
    tight, wide = (b.grads(r, p.scale, 2, p.bucket, p.reach, p.buckets, 2.0 ** -24, x) for x in (True, False))
    q, k = (at % 128 < 3)[:, None], ((at % 128 < 3) | (at % 128 >= 125))[:, None]
    near(p.heads(p.dQ, 4), r["dQ"], torch.where(q, wide["dQ"], tight["dQ"]), "dQ")
    near(p.heads(p.dK, 2), r["dK"], torch.where(k, wide["dK"], tight["dK"]), "dK")
    near(p.dtable, r["dtable"], wide["dtable"], "dtable")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cap", [1e3, 3e3, 2e4, 1e6, 1e9, 1e30])
def test_large_caps(dev, cap, dtype):
    """Caps that hardly bend the scores cost them no digits: the bounds are those of scores without a cap."""
    p = Problem(dev, 1, 200, 2, 1, 64, dtype, "causal", cap, sigma=2.0)
    check_forward(p)
    f = p.exact()
    b = Bounds(f, dtype, p.T, p.hd, 0.0, None)
    near(p.heads(p.O, p.H), f["o"], b.o(), "O")
    near(p.lse, f["lse"], b.lse(), "lse")
    check_backward(p, f, b)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cap,buckets,slope", [(0.0, 0, False), (30.0, 6, False), (50.0, 0, False), (90.0, 6, False), (20.0, 0, True)])
def test_single_keys(dev, cap, buckets, slope, dtype):
    """A token that sees one key has that key's value, to the last bit; one key of the other half of a tile of keys among them."""
    p = Problem(dev, 2, 200, 4, 2, 64, dtype, "full", cap, buckets, 30 if buckets else 0, slope, sigma=2.0)
    key = torch.randint(0, 200, (2, 200), generator=torch.Generator().manual_seed(4)).to(dev)
    p.range = torch.stack([key, key + 1], 2).int().contiguous()
    p.seen = torch.arange(200, device=dev) == key[..., None]
    f, b = check_forward(p)
    v = p.heads(p.V, 2).repeat_interleave(2, 1).gather(2, key[:, None, :, None].expand(2, 4, 200, 64))
    assert torch.equal(p.heads(p.O, 4), v)
    check_backward(p, f, b)
    assert (p.dQ == 0).all() and (p.dK == 0).all()


MORE = [
    ((12, 300, 16, 4, 128), "docs", 20.0, 32, 128, True),   # items over several rounds, a row of scores over two warps
    ((40, 129, 8, 8, 64), "any", 5.0, 300, 60, False),
    ((1, 1300, 2, 1, 64), "causal", 0.0, 1024, 2000, False),  # distances that are summed by bucket
    ((2, 700, 4, 2, 128), "docs", 30.0, 600, 699, True),
    ((1, 600, 2, 2, 40), "full", 0.0, 33, 560, False),
    ((1, 1500, 3, 3, 64), "window", 50.0, 2, 0, False),       # one distance for all
    ((1, 150, 32, 4, 64), "causal", 20.0, 1024, 140, False),  # a table that no CTA reads beforehand
]


@pytest.mark.parametrize("shape,mask,cap,buckets,reach,slope", MORE)
def test_many_items_and_wide_tables(dev, shape, mask, cap, buckets, reach, slope):
    p = Problem(dev, *shape, BF, mask, cap, buckets, reach, slope)
    f, b = check_forward(p)
    check_backward(p, f, b, beta=0.5, grad=F32)


@pytest.mark.parametrize("mask", ["causal", "any"])
def test_long(dev, mask):
    p = Problem(dev, 1, 6001, 2, 1, 64, BF, mask)
    f, b = check_forward(p)
    check_backward(p, f, b)


@pytest.mark.parametrize("dtype,hd", [(BF, 64), (BF, 28), (F32, 64)])
def test_offsets_past_32_bits(dev, dtype, hd):
    """Rows 2^25 bytes and more apart: the last ones lie past 2^32 bytes, with 130 rows past 2^31 values."""
    p = Problem(dev, 2, 65, 1, 1, hd, dtype, "docs", layout=((1 << 24) + 64 - hd, 8))
    f, b = check_forward(p)
    check_backward(p, f, b)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_wild_ranges(dev, dtype):
    """Ranges with ends anywhere in 32 bits are clamped."""
    p = Problem(dev, 2, 200, 2, 1, 64, dtype, "full")
    g = torch.Generator().manual_seed(3)
    ends = torch.tensor([-2 ** 31, -2 ** 31 + 1, -1, 0, 1, 63, 64, 128, 199, 200, 201, 2 ** 31 - 2, 2 ** 31 - 1])
    p.range = ends[torch.randint(0, len(ends), (2, 200, 2), generator=g)].int().to(dev)
    p.L.causal = 1  # not read
    at = torch.arange(200, device=dev)
    p.seen = (at >= p.range[..., :1]) & (at < p.range[..., 1:])
    f, b = check_forward(p)
    check_backward(p, f, b)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_one_tensor_for_all(dev, dtype):
    p = Problem(dev, 2, 150, 2, 2, 64, dtype, "causal")
    p.K = p.V = p.Q
    f, b = check_forward(p)
    check_backward(p, f, b)


def test_two_calls_at_once(dev):
    """Two batches on two streams, each with its workspace, as calls and as graphs, many times over each other."""
    ps = [Problem(dev, 3, 700, 8, 2, 64, BF, "docs", 20.0, 16, 64, seed=s) for s in (1, 2)]
    names = ("O", "lse", "dQ", "dK", "dV", "dtable")
    want = []
    for p in ps:
        p.forward()
        p.backward()
        want.append([getattr(p, x).clone() for x in names])
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(5):
        for p, s in zip(ps, streams):
            with torch.cuda.stream(s):
                p.forward()
                p.backward()
    torch.cuda.synchronize()
    for p, w in zip(ps, want):
        assert all(torch.equal(getattr(p, x), y) for x, y in zip(names, w))
    graphs = []
    for p in ps:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            p.forward()
            p.backward()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    tda.tda_device_status()
    torch.cuda.synchronize()
    for p, w in zip(ps, want):
        assert all(torch.equal(getattr(p, x), y) for x, y in zip(names, w))


def test_warps_that_run_ahead(dev):
    """Pairs of tiles with diagonals to sum beside pairs without: the fast warps' weights never stand in for the slow ones'."""
    p = Problem(dev, 1, 700, 4, 1, 64, BF, "full", 30.0, 5, 40, sigma=4.0)
    f, b = check_forward(p)
    for _ in range(40):
        check_backward(p, f, b)


def test_no_lse_and_empty_batches(dev):
    p = Problem(dev, 1, 90, 2, 1, 64, BF, "causal")
    p.forward()
    with_lse = p.O.clone()
    wsb = tda.tda_attention_workspace_size(tda.TDA_ATTENTION_FORWARD, p.L)
    ws = torch.empty(max(wsb, 1), dtype=torch.uint8, device=dev)
    tda.tda_attention_forward(p.L, p.Q, p.Q.stride(0), p.K, p.K.stride(0), p.V, p.V.stride(0), None, None, None, None, p.O,
                              p.O.stride(0), None, ws, wsb)
    assert torch.equal(p.O, with_lse)
    for N, T in ((0, 5), (3, 0)):
        L = tda.AttentionDesc(N, T, 2, 1, 64, n_buckets=4, max_distance=8)
        table = torch.full((4, 2), 3.0, device=dev)
        tda.tda_attention_forward(L, None, 128, None, 64, None, 64, None, None, None, None, None, 128)
        tda.tda_attention_backward(L, None, 128, None, 64, None, 64, None, None, None, None, None, 128, None, None, 128, None, 128,
                                   None, 64, None, 64, table, tda.TDA_F32, 0.5)
        assert (table == 1.5).all()


def test_streams_and_graphs(dev):
    """On another stream than the current one, and captured with the backward pass and replayed on new inputs."""
    p = Problem(dev, 2, 300, 4, 2, 64, BF, "docs", 20.0, 16, 64)
    p.forward()
    p.backward()
    want = [x.clone() for x in (p.O, p.lse, p.dQ, p.dK, p.dV, p.dtable)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    p.forward(s)
    p.backward(stream=s)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, (p.O, p.lse, p.dQ, p.dK, p.dV, p.dtable)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.forward()
        p.backward()
    kept = (p.O, p.lse, p.dQ, p.dK, p.dV, p.dtable)
    p.buf.copy_(torch.where(torch.isfinite(p.buf.float()), -p.buf, p.buf))  # other queries, keys, values
    graph.replay()
    tda.tda_device_status()
    got = [x.clone() for x in kept]
    p.forward()
    p.backward()
    assert all(torch.equal(x, y) for x, y in zip(got, (p.O, p.lse, p.dQ, p.dK, p.dV, p.dtable)))
    assert not torch.equal(got[0], want[0])


# ------------------------------------------------------------------ ranges
def by_hand(doc, pre, causal, window):
    N, T = doc.shape
    out = torch.zeros((N, T, 2), dtype=torch.int32)
    for n in range(N):
        d, f = doc[n].tolist(), pre[n].tolist()
        s = 0
        while s < T:
            e = s
            while e < T and d[e] == d[s]:
                e += 1
            p = s
            while p < e and f[p]:
                p += 1
            for i in range(s, e):
                lo, hi = s, max(i + 1, p) if causal else e
                if window:
                    lo, hi = max(lo, i - window + 1), min(hi, i + window)
                out[n, i] = torch.tensor([lo, hi]) if d[s] >= 0 else 0
            s = e
    return out


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("N,T,docs,window", [(1, 1, 1, 0), (3, 7, 2, 0), (2, 33, 5, 4), (1, 1000, 9, 0), (2, 8192, 30, 511),
                                             (1, 8193, 3, 0), (2, 20001, 400, 0), (1, 30000, 2, 9000)])
def test_ranges(dev, N, T, docs, window, causal):
    gen = torch.Generator().manual_seed(T + docs)
    doc = (torch.rand((N, T), generator=gen) < docs / T).int().cumsum(1).int()
    doc[torch.rand((N, T), generator=gen) < 0.01] = -1
    doc[:, T - T // 9:] = -5
    pre = (torch.rand((N, T), generator=gen) < 0.97).int() * 3
    out = torch.full((N * T + 1, 2), 7, dtype=torch.int32, device=dev)
    none = torch.zeros_like(pre)
    for d, p in ((doc, pre), (doc, None), (None, pre), (None, None)):
        tda.tda_attention_ranges(N, T, None if d is None else d.to(dev), None if p is None else p.to(dev), causal, window, out)
        want = by_hand(none if d is None else d, none if p is None else p, causal, window)
        assert torch.equal(out[:N * T].cpu(), want.view(N * T, 2)) and (out[N * T] == 7).all()


def test_bucket_gradient_is_a_difference(dev):
    """dtable against central differences of the fp32 forward pass along a direction of the table."""
    p = Problem(dev, 1, 96, 2, 1, 32, F32, "causal", 4.0, 6, 40)
    p.forward()
    p.backward()
    got = p.dtable.double()
    step = torch.randn(6, 2, device=dev, dtype=torch.float64)
    table, h = p.table.double(), 1e-5
    out = []
    for sign in (1, -1):
        b = bias_of(96, 2, p.bucket, 40, table + sign * h * step, None, dev)
        out.append((attention(p.heads(p.Q, 2), p.heads(p.K, 1), p.heads(p.V, 1), p.seen, p.scale, 4.0, b)["o"]
                    * p.heads(p.dO, 2).double()).sum())
    want = (out[0] - out[1]) / (2 * h)
    # third order of the difference h^2, 64-bit rounding 1e-16 / h; the kernel's fp32 sums 2^-24 (96 + 32) per term
    size = by_bucket(gradients(p.exact(), p.heads(p.dO, 2), p.scale, 1)["ds"].abs(), p.bucket, 40, 6)
    assert ((got * step).sum() - want).abs() <= 2.0 ** -15 * (size * step.abs()).sum() + 1e-6
