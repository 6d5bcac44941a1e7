"""Host validation of the attention's and the norm's entry points, the map of distances to buckets, and the 64-bit
reference against differences (no GPU: a refused call launches nothing)."""
import ctypes
import math

import pytest
import torch

import paper_2609_38767_gb300 as tda
from attention_reference import attention, bias_of, gradients, seen_by
from paper_2609_38767_gb300 import build as tbuild

BAD, UNSUPPORTED, WORKSPACE = tda.TDA_ERR_INVALID_ARG, tda.TDA_ERR_UNSUPPORTED, tda.TDA_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def libs():
    return tbuild.build()


def err(fn, *a, **k):
    with pytest.raises(tda.TdaError) as e:
        fn(*a, stream=0, **k)
    assert str(e.value)
    return e.value.status


def desc(N=2, T=40, heads=4, kv_heads=2, head_dim=64, dtype=tda.TDA_BF16, scale=0.1, cap=0.0, causal=1, n_buckets=0, max_distance=0):
    L = tda.AttentionDesc(N, T, heads, kv_heads, head_dim, dtype, scale, cap, True, n_buckets, max_distance)
    L.causal = causal
    return L


BAD_DESCS = [dict(N=-1), dict(T=-1), dict(N=1 << 31), dict(T=1 << 31), dict(N=1, T=(1 << 29) + 1, heads=1, kv_heads=1), dict(N=1 << 20, T=1 << 20), dict(heads=0), dict(kv_heads=0),
             dict(kv_heads=3), dict(heads=65536, kv_heads=1), dict(head_dim=0), dict(dtype=tda.TDA_F64), dict(dtype=7),
             dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(cap=-1.0), dict(cap=math.nan),
             dict(cap=math.inf), dict(causal=2), dict(causal=-1), dict(n_buckets=-1), dict(n_buckets=1025), dict(max_distance=-1),
             dict(max_distance=(1 << 20) + 1), dict(N=1 << 16, T=1 << 14, heads=4096, kv_heads=1),
             dict(N=1 << 14, T=1, heads=65535, kv_heads=1)]


def fwd(L=None, Q=256, ld_q=256, K=256, ld_k=128, V=256, ld_v=128, rng=None, bucket=None, table=None, slope=None, O=256, ld_o=256,
        lse=None, ws=None, wsb=0):
    return err(tda.tda_attention_forward, L or desc(), Q, ld_q, K, ld_k, V, ld_v, rng, bucket, table, slope, O, ld_o, lse, ws, wsb)


def bwd(L=None, Q=256, ld_q=256, K=256, ld_k=128, V=256, ld_v=128, rng=None, bucket=None, table=None, slope=None, O=256, ld_o=256,
        lse=256, dO=256, ld_do=256, dQ=256, ld_dq=256, dK=256, ld_dk=128, dV=256, ld_dv=128, dtable=None, gt=tda.TDA_F32, beta=0.0,
        ws=256, wsb=1 << 30):
    return err(tda.tda_attention_backward, L or desc(), Q, ld_q, K, ld_k, V, ld_v, rng, bucket, table, slope, O, ld_o, lse, dO,
               ld_do, dQ, ld_dq, dK, ld_dk, dV, ld_dv, dtable, gt, beta, ws, wsb)


def test_attention_descriptor():
    assert ctypes.sizeof(tda.AttentionDesc) == 56 and tda.AttentionDesc.max_distance.offset == 48
    for k in BAD_DESCS:
        assert fwd(desc(**k)) == BAD and bwd(desc(**k)) == BAD, k
        for op in (tda.TDA_ATTENTION_FORWARD, tda.TDA_ATTENTION_BACKWARD):
            with pytest.raises(tda.TdaError):
                tda.tda_attention_workspace_size(op, desc(**k))
    assert fwd(desc(head_dim=129)) == UNSUPPORTED and fwd(desc(head_dim=1 << 20)) == UNSUPPORTED
    with pytest.raises(tda.TdaError):
        tda.tda_attention_workspace_size(2, desc())
    for N, T, h in ((1, 1 << 29, 3), (1 << 20, 1 << 9, 3), (1 << 13, 1, 65535)):  # the largest that fit in 32 bits
        for op in (tda.TDA_ATTENTION_FORWARD, tda.TDA_ATTENTION_BACKWARD):
            assert tda.tda_attention_workspace_size(op, desc(N=N, T=T, heads=h, kv_heads=h)) > 0
    for N, T in ((0, 40), (2, 0)):  # nothing to do
        tda.tda_attention_forward(desc(N=N, T=T), None, 0, None, 0, None, 0, None, None, None, None, None, 0, stream=0)
        assert tda.tda_attention_workspace_size(tda.TDA_ATTENTION_BACKWARD, desc(N=N, T=T)) == 0


def test_the_attention_is_an_attention_descriptor():
    for other in (b"", bytes(desc()), bytearray(56), tda.LinearDesc(64, 32), memoryview(desc())):
        with pytest.raises(TypeError):
            tda.tda_attention_forward(other, 256, 256, 256, 128, 256, 128, None, None, None, None, 256, 256, stream=0)
        with pytest.raises(TypeError):
            tda.tda_attention_backward(other, 256, 256, 256, 128, 256, 128, None, None, None, None, 256, 256, 256, 256, 256, 256,
                                       256, 256, 128, 256, 128, stream=0)


def test_attention_refusals():
    shared = [dict(Q=None), dict(K=None), dict(V=None), dict(Q=257), dict(K=257), dict(V=257), dict(ld_q=255), dict(ld_k=127),
              dict(ld_v=127), dict(ld_q=1 << 40), dict(rng=260), dict(slope=258), dict(O=None), dict(O=257), dict(ld_o=255),
              dict(lse=258)]
    learned = [dict(), dict(bucket=256), dict(table=256), dict(bucket=258, table=256), dict(bucket=256, table=257)]
    for call in (fwd, bwd):
        for k in shared:
            assert call(**k) == BAD, k
        for k in learned:
            assert call(desc(n_buckets=4, max_distance=9), **k) == BAD, k
    for k in (dict(lse=None), dict(dO=None), dict(dO=257), dict(ld_do=255), dict(dQ=None), dict(dQ=257), dict(ld_dq=255),
              dict(dK=None), dict(dK=257), dict(ld_dk=127), dict(dV=None), dict(dV=257), dict(ld_dv=127), dict(gt=tda.TDA_F64),
              dict(gt=9), dict(beta=math.nan), dict(beta=math.inf), dict(dtable=256), dict(ws=257),
              dict(L=desc(n_buckets=4), bucket=256, table=256, dtable=258)):
        assert bwd(**k) == BAD, k
    assert bwd(desc(dtype=tda.TDA_F32), gt=tda.TDA_BF16) == UNSUPPORTED
    need = tda.tda_attention_workspace_size(tda.TDA_ATTENTION_BACKWARD, desc())
    assert need > 0 and bwd(wsb=256) == WORKSPACE and bwd(ws=None) == WORKSPACE
    for call in (lambda b: fwd(ws=256, wsb=b), lambda b: bwd(wsb=b)):
        with pytest.raises(OverflowError):
            call(-1)


def test_ranges_refusals():
    def rng(N=2, T=9, doc=256, prefix=256, causal=1, window=0, out=256):
        return err(tda.tda_attention_ranges, N, T, doc, prefix, causal, window, out)

    for k in (dict(N=-1), dict(T=-1), dict(N=1 << 31), dict(T=1 << 31), dict(N=1 << 20, T=1 << 20), dict(doc=257), dict(prefix=258),
              dict(causal=2), dict(window=-1), dict(window=1 << 31), dict(out=None), dict(out=260)):
        assert rng(**k) == BAD, k
    tda.tda_attention_ranges(0, 9, None, None, 1, 0, None, stream=0)
    tda.tda_attention_ranges(9, 0, None, None, 1, 0, None, stream=0)


def test_norm_refusals():
    def f(dtype=tda.TDA_BF16, x=256, ld_x=64, r=256, ld_r=64, M=3, d=64, w=256, eps=1e-5, h=256, ld_h=64, y=256, ld_y=64, rstd=256):
        return err(tda.tda_rmsnorm_forward, dtype, x, ld_x, r, ld_r, M, d, w, eps, h, ld_h, y, ld_y, rstd)

    for k in (dict(dtype=tda.TDA_F64), dict(M=-1), dict(M=1 << 31), dict(d=0), dict(x=None), dict(x=257), dict(ld_x=63), dict(r=257),
              dict(ld_r=63), dict(w=None), dict(w=257), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf),
              dict(h=257), dict(ld_h=63), dict(y=None), dict(y=257), dict(ld_y=63), dict(rstd=258)):
        assert f(**k) == BAD, k
    assert f(d=32769, ld_x=40000) == UNSUPPORTED
    tda.tda_rmsnorm_forward(tda.TDA_F32, None, 0, None, 0, 0, 64, None, 1e-5, None, 0, None, 0, stream=0)

    def b(dtype=tda.TDA_BF16, h=256, ld_h=64, rstd=256, w=256, dy=256, ld_dy=64, dres=256, ld_r=64, M=3, d=64, dx=256, ld_dx=64, dw=256,
          gt=tda.TDA_F32, beta=0.0, ws=256, wsb=1 << 20):
        return err(tda.tda_rmsnorm_backward, dtype, h, ld_h, rstd, w, dy, ld_dy, dres, ld_r, M, d, dx, ld_dx, dw, gt, beta, ws, wsb)

    for k in (dict(dtype=tda.TDA_F64), dict(M=-1), dict(d=0), dict(h=None), dict(h=257), dict(ld_h=63), dict(rstd=None), dict(rstd=258),
              dict(w=None), dict(dy=None), dict(dy=257), dict(ld_dy=63), dict(dres=257), dict(ld_r=63), dict(dx=257), dict(ld_dx=63),
              dict(dw=258), dict(gt=tda.TDA_F64), dict(beta=math.nan), dict(ws=264)):
        assert b(**k) == BAD, k
    assert b(dtype=tda.TDA_F32, gt=tda.TDA_BF16) == UNSUPPORTED and b(d=40000, ld_h=40000) == UNSUPPORTED
    need = tda.tda_rmsnorm_workspace_size(3, 64)
    assert need > 0 and b(wsb=need - 1) == WORKSPACE and b(ws=None) == WORKSPACE
    assert tda.tda_rmsnorm_workspace_size(0, 64) == 0 and tda.tda_rmsnorm_workspace_size(3, 32769) == 0
    with pytest.raises(OverflowError):
        b(wsb=-1)


@pytest.mark.parametrize("n,reach,both", [(2, 2, 0), (4, 2, 1), (32, 128, 1), (32, 128, 0), (16, 300, 0), (1024, 5000, 1), (7, 40, 0)])
def test_position_buckets(n, reach, both):
    out = torch.full((2 * reach + 2,), 77, dtype=torch.int32)
    tda.tda_position_buckets(n, reach, both, out)
    side = n // 2 if both else n
    e = side // 2
    for d in range(-reach, reach + 1):
        a = abs(d) if both else max(d, 0)
        if a < e:
            want = a
        else:  # the largest k with e (reach / e)^(k / (side - e)) <= a, in whole numbers
            k = 0
            while k < side - e - 1 and e ** (side - e) * reach ** (k + 1) <= a ** (side - e) * e ** (k + 1):
                k += 1
            want = e + k
        assert out[d + reach] == want + (side if both and d < 0 else 0), d
    assert out[2 * reach + 1] == 77
    for bad in ((1, 9, 0), (2, 9, 1), (5, 9, 1), (1025, 3000, 0), (8, 4, 0), (8, (1 << 20) + 1, 0), (8, 9, 2)):
        with pytest.raises(tda.TdaError):
            tda.tda_position_buckets(*bad, 256)
    for short in (torch.zeros(2 * reach, dtype=torch.int32), torch.zeros(2 * reach + 1), torch.zeros(4 * reach + 2, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            tda.tda_position_buckets(n, reach, both, short)


def test_reference_gradients_are_differences():
    """The 64-bit reference that the kernels are compared with, against central differences of its forward pass."""
    g = torch.Generator().manual_seed(3)
    N, T, H, KV, d, cap, n, reach = 2, 11, 4, 2, 5, 1.5, 3, 6
    q, k, v = (torch.randn((N, h, T, d), generator=g, dtype=torch.float64) for h in (H, KV, KV))
    table, do = torch.randn((n, H), generator=g, dtype=torch.float64), torch.randn((N, H, T, d), generator=g, dtype=torch.float64)
    bucket = torch.randint(-1, n + 1, (2 * reach + 1,), generator=g)
    slope = torch.rand(H, generator=g, dtype=torch.float64)
    at = torch.arange(T).expand(N, T)
    rng = torch.stack([(at - 4).clamp(min=-1), at + 2], 2)
    rng[0, 3] = 0
    rng[1, 2:4, 1] = rng[1, 2:4, 0] + 1
    seen = seen_by(rng, T, N, False, "cpu")

    def loss(q, k, v, table):
        return (attention(q, k, v, seen, 0.4, cap, bias_of(T, H, bucket, reach, table, slope, "cpu"))["o"] * do).sum()

    f = attention(q, k, v, seen, 0.4, cap, bias_of(T, H, bucket, reach, table, slope, "cpu"))
    r = gradients(f, do, 0.4, KV, bucket, reach, n)
    args, h = [q, k, v, table], 1e-5
    for i, name in enumerate(("dQ", "dK", "dV", "dtable")):
        for _ in range(4):
            step = torch.randn(args[i].shape, generator=g, dtype=torch.float64)
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + h * step, args[i] - h * step
            diff = (loss(*up) - loss(*down)) / (2 * h)
            assert abs(diff - (r[name] * step).sum()) <= 1e-6 * (1 + abs(diff)), name
