"""Host validation of the training step's entry points (no GPU: a refused call launches nothing)."""
import ctypes

import pytest
import torch

import paper_2609_38767_gb300 as tda
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


def forward(dtype=tda.TDA_BF16, E=256, ld_e=8, V=4, d=8, it=tda.TDA_I32, tok=256, n=3, scale=1.0, out=256, ld_out=8):
    return err(tda.tda_embedding_forward, dtype, E, ld_e, V, d, it, tok, n, scale, out, ld_out)


def test_embedding_forward_refusals():
    for k in (dict(dtype=tda.TDA_F64), dict(dtype=9), dict(E=None), dict(E=257), dict(out=None), dict(out=255),
              dict(ld_e=7), dict(ld_out=7), dict(V=0), dict(V=1 << 31), dict(d=0), dict(n=-1), dict(n=1 << 31),
              dict(it=2), dict(tok=None), dict(tok=258), dict(it=tda.TDA_I64, tok=260), dict(scale=float("nan")),
              dict(scale=float("inf"))):
        assert forward(**k) == BAD, k
    tda.tda_embedding_forward(tda.TDA_F32, None, 8, 4, 8, tda.TDA_I32, None, 0, 1.0, None, 8, stream=0)  # no tokens


def backward(dtype=tda.TDA_BF16, dout=256, ld_d=8, V=4, d=8, it=tda.TDA_I32, tok=256, n=3, scale=1.0,
             gt=tda.TDA_F32, dE=256, ld_e=8, beta=0.0, ws=256, wsb=1 << 20):
    return err(tda.tda_embedding_backward, dtype, dout, ld_d, V, d, it, tok, n, scale, gt, dE, ld_e, beta, ws, wsb)


def test_embedding_backward_refusals():
    for k in (dict(dtype=tda.TDA_F64), dict(gt=tda.TDA_F64), dict(dout=None), dict(dout=257), dict(dE=None),
              dict(dE=258), dict(ld_d=7), dict(ld_e=7), dict(V=0), dict(d=0), dict(n=-1), dict(it=-1), dict(tok=None),
              dict(scale=float("inf")), dict(beta=float("nan")), dict(ws=257)):
        assert backward(**k) == BAD, k
    assert backward(dtype=tda.TDA_F32, gt=tda.TDA_BF16) == UNSUPPORTED
    need = tda.tda_embedding_workspace_size(4, 8, 3)
    assert need > 0
    assert backward(wsb=need - 1) == WORKSPACE and backward(ws=None) == WORKSPACE
    assert tda.tda_embedding_workspace_size(4, 8, 0) == 0 and tda.tda_embedding_workspace_size(0, 8, 3) == 0


def ref(in_=256, out=256, n=4, dtype=tda.TDA_F32):
    return (tda.TensorRef * 1)(tda.TensorRef(in_, out, n, dtype, 0))


def test_grad_clip_refusals():
    assert ctypes.sizeof(tda.TensorRef) == 32
    wsb = tda.tda_grad_clip_workspace_size(ref(), 1)
    assert wsb > 0 and tda.tda_grad_clip_workspace_size(ref(), -1) == 0

    def clip(refs=None, n=1, max_norm=1.0, norm=256, ws=256, b=wsb):
        return err(tda.tda_grad_clip, refs if refs is not None else ref(), n, max_norm, norm, ws, b)

    for k in (dict(n=-1), dict(n=1 << 21), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")),
              dict(norm=None), dict(norm=257), dict(refs=ref(dtype=tda.TDA_F64)), dict(refs=ref(n=-1)),
              dict(refs=ref(in_=None)), dict(refs=ref(in_=258)), dict(refs=ref(out=257, dtype=tda.TDA_BF16)),
              dict(ws=264)):
        assert clip(**k) == BAD, k
    assert clip(b=wsb - 1) == WORKSPACE and clip(ws=None) == WORKSPACE


def test_tensor_list_refusals():
    a = torch.zeros(4, 6)
    for ts, outs in (([a.t()], None), ([a.double()], None), ([a], [a, a]), ([a], [a.bfloat16()]), ([a], [a[:2]]),
                     ([a], [a.t()])):
        with pytest.raises(ValueError):
            tda.tensor_list(ts, outs)
    refs = tda.tensor_list([a, a.bfloat16()], [None, None])
    assert refs[0].n == 24 and refs[0].out is None and refs[1].dtype == tda.TDA_BF16


def layer(d_in=64, d_out=32, act=0, dtype=tda.TDA_BF16):
    return tda.LinearDesc(d_in, d_out, act, dtype)


def test_linear_descriptor_and_workspace():
    assert ctypes.sizeof(tda.LinearDesc) == 24
    F, B, ANY = tda.TDA_LINEAR_FORWARD, tda.TDA_LINEAR_BACKWARD, tda.TDA_LINEAR_ANY_STRIDE
    size = tda.tda_linear_workspace_size
    assert size(F, layer(), 10) == 0 and size(F, layer(), 0) == 0
    assert size(F | ANY, layer(), 10) >= 2 * 64 * (10 + 32)
    assert size(F, layer(d_in=65), 10) >= 2 * 72 * (10 + 32)  # rows of 65 values need aligned copies
    assert size(F, layer(dtype=tda.TDA_F32), 10) >= 6 * 64 * (10 + 32)
    assert size(B, layer(), 10) >= 4 * 32
    for bad in (lambda: size(7, layer(), 1), lambda: size(F, layer(d_in=0), 1), lambda: size(F, layer(), -1),
                lambda: size(F, layer(act=5), 1), lambda: size(F, layer(dtype=tda.TDA_F64), 1)):
        with pytest.raises(tda.TdaError):
            bad()


def test_linear_forward_refusals():
    def fwd(L=None, X=256, ld_x=64, M=40, W=256, ld_w=64, bias=None, R=None, ld_r=32, Y=256, ld_y=32, Z=None, ld_z=32,
            ws=None, wsb=0):
        return err(tda.tda_linear_forward, L or layer(), X, ld_x, M, W, ld_w, bias, R, ld_r, Y, ld_y, Z, ld_z, ws, wsb)

    for k in (dict(L=layer(d_out=0)), dict(L=layer(act=-1)), dict(L=layer(dtype=2)), dict(M=-1), dict(M=1 << 31),
              dict(X=None), dict(X=257), dict(ld_x=63), dict(W=None), dict(ld_w=63), dict(bias=257), dict(R=257),
              dict(R=256, ld_r=31), dict(Y=None), dict(Y=255), dict(ld_y=31), dict(Z=255), dict(Z=256, ld_z=31),
              dict(ld_x=1 << 40)):
        assert fwd(**k) == BAD, k
    f32 = layer(dtype=tda.TDA_F32)
    need = tda.tda_linear_workspace_size(tda.TDA_LINEAR_FORWARD, f32, 40)
    assert fwd(L=f32, ws=256, wsb=need - 1) == WORKSPACE and fwd(L=f32) == WORKSPACE
    assert fwd(L=f32, ws=264, wsb=need) == BAD
    assert fwd(ld_x=65) == WORKSPACE  # rows off 16 bytes need a copy


def test_linear_backward_refusals():
    def bwd(L=None, dY=256, ld_dy=32, Z=256, ld_z=32, M=4, X=256, ld_x=64, W=256, ld_w=64, B=256, ld_b=32, dX=256,
            ld_dx=64, dW=256, ld_dw=64, db=256, gt=tda.TDA_F32, beta=0.0, ws=256, wsb=1 << 20):
        return err(tda.tda_linear_backward, L or layer(act=tda.TDA_ACT_SILU), dY, ld_dy, Z, ld_z, M, X, ld_x, W, ld_w, B,
                   ld_b, dX, ld_dx, dW, ld_dw, db, gt, beta, ws, wsb)

    for k in (dict(dY=None), dict(dY=257), dict(ld_dy=31), dict(Z=None), dict(ld_z=31), dict(B=None), dict(B=257),
              dict(ld_b=31), dict(X=None), dict(W=None), dict(ld_w=63), dict(dX=257), dict(ld_dx=63), dict(dW=258),
              dict(ld_dw=63), dict(db=257), dict(gt=tda.TDA_F64), dict(beta=float("inf")), dict(M=-1), dict(ws=264)):
        assert bwd(**k) == BAD, k
    assert bwd(L=layer(act=1, dtype=tda.TDA_F32), gt=tda.TDA_BF16) == UNSUPPORTED
    assert bwd(wsb=100) == WORKSPACE and bwd(ws=None) == WORKSPACE


def test_calls_with_arguments_of_the_wrong_kind():
    """The binding converts before it calls: a Python error, and nothing reaches the library."""
    for bad in (dict(E="x"), dict(ld_e=1.5), dict(n=None), dict(scale="a"), dict(tok=object()), dict(V=1 << 70)):
        k = dict(dtype=tda.TDA_BF16, E=256, ld_e=8, V=4, d=8, it=tda.TDA_I32, tok=256, n=3, scale=1.0, out=256, ld_out=8)
        k.update(bad)
        with pytest.raises((TypeError, AttributeError, OverflowError)):
            tda.tda_embedding_forward(*k.values(), stream=0)
    with pytest.raises(TypeError):
        tda.tda_linear_forward(3, 256, 64, 1, 256, 64, None, None, 0, 256, 32, stream=0)
    with pytest.raises(ValueError):  # more tensors than the list holds
        tda.tda_grad_clip(ref(), 2, 1.0, 256, 256, 1 << 20, stream=0)
    with pytest.raises(tda.TdaError):  # no descriptor: the library's own refusal
        tda.tda_linear_forward(None, 256, 64, 1, 256, 64, None, None, 0, 256, 32, stream=0)
