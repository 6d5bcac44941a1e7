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
