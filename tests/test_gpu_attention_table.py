"""The gradient of a learned position bias in long examples, to the bounds of attention_table."""
import pytest
import torch

import paper_2609_38767_gb300 as tda
from attention_reference import Bounds, bias_of, gradients
from attention_table import table_bound
from paper_2609_38767_gb300 import build as tbuild
from test_gpu_attention import BF, F32, MORE, Problem, check_backward, check_forward, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


def toward_values(p):
    """dO of a token along its own value, so that its own pair gains and the sum of dS along the diagonal is large and positive."""
    v = p.heads(p.V, p.KV).repeat_interleave(p.H // p.KV, 1)
    p.dO.copy_(v.transpose(1, 2).reshape(p.N * p.T, p.H * p.hd))


def check_table(p):
    """dtable within its bound; the exact dS and the bound."""
    p.forward()
    p.backward(grad=F32)
    tda.tda_device_status()
    f = p.exact()
    b = Bounds(f, p.dtype, p.T, p.hd, p.cap, p.bias)
    r = gradients(f, p.heads(p.dO, p.H), p.scale, p.KV, p.bucket, p.reach, p.buckets)
    tol = table_bound(f, b, r, p.bucket, p.reach, p.buckets, 2.0 ** -24)
    near(p.dtable, r["dtable"], tol, "dtable")
    return r["ds"], tol


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,T,H,KV,hd,mask,cap,buckets,bucket", [
    (1, 100, 2, 2, 64, "causal", 0.0, 1, 0), (1, 1500, 3, 3, 64, "window", 50.0, 2, 0), (2, 700, 4, 2, 128, "full", 0.0, 3, 2),
    (1, 1000, 2, 1, 64, "causal", 30.0, 1, 0), (3, 130, 4, 4, 80, "docs", 20.0, 2, 1), (1, 300, 2, 2, 64, "causal", 0.0, 2, -1)])
def test_one_bucket_for_all_distances(dev, N, T, H, KV, hd, mask, cap, buckets, bucket, dtype):
    """max_distance = 0: all pairs share a bias, which changes nothing, so its gradient is 0; a bucket that does not exist has none."""
    p = Problem(dev, N, T, H, KV, hd, dtype, mask, cap, buckets, 0, garbage=False)
    p.bucket = torch.full((1,), bucket, dtype=torch.int32, device=dev)
    p.bias = bias_of(T, H, p.bucket, 0, p.table, None, dev)
    toward_values(p)
    ds, tol = check_table(p)
    diagonal = ds.diagonal(dim1=2, dim2=3).sum((0, 2))
    if bucket >= 0:
        assert (diagonal > 4 * tol[bucket]).all()  # what a diagonal counted twice or not at all leaves
        p.dtable[bucket] = 0
    assert (p.dtable == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape,mask,cap,buckets,reach,slope", MORE + [
    ((2, 1030, 4, 1, 64), "docs", 30.0, 32, 128, False), ((1, 2000, 2, 2, 128), "full", 0.0, 40, 511, False),
    ((1, 1100, 4, 2, 64), "any", 50.0, 12, 300, True)])
def test_long_examples(dev, shape, mask, cap, buckets, reach, slope, dtype):
    p = Problem(dev, *shape, dtype, mask, cap, buckets, reach, slope)
    toward_values(p)
    idle = ~p.seen.any(2).reshape(-1)
    p.dO[idle] = float("nan")
    check_table(p)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hd,cap,buckets", [(64, 0.0, 0), (128, 30.0, 16), (64, 0.0, 16)])
def test_causal_order_as_ranges(dev, hd, cap, buckets, dtype):
    """Keys up to the token itself, said by ranges."""
    p = Problem(dev, 2, 450, 4, 2, hd, dtype, "causal_range", cap, buckets, 60 if buckets else 0)
    f, b = check_forward(p)
    check_backward(p, f, b)
    got = [x.clone() for x in (p.O, p.lse, p.dQ, p.dK, p.dV)]
    p.range, p.L.causal = None, 1
    f, b = check_forward(p)
    check_backward(p, f, b)
    for x, y in zip(got, (p.O, p.lse, p.dQ, p.dK, p.dV)):
        assert torch.equal(x, y)  # the same tiles in the same order
