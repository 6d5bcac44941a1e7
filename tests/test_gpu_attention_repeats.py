"""Attention whose rows' bases move from tile to tile of keys: within the bounds of attention_reference.Bounds, and equal bits
from many equal calls."""
import math

import pytest
import torch

import paper_2609_38767_gb300 as tda
from attention_reference import bias_of
from paper_2609_38767_gb300 import build as tbuild
from test_gpu_attention import BF, F32, Problem, check_backward, check_forward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


def at_the_cap(dev, cap, buckets, hd):
    """Capped scores that rise and fall from one end of their range to the other, of heads in directions of their own."""
    T = 700
    p = Problem(dev, 1, T, 4, 1, hd, BF, "full", cap, buckets, 40 if buckets else 0, sigma=0.5)
    at = torch.arange(T, device=dev)
    along = torch.stack([torch.sin(at / 40.0) * 3, at / T * 6 - 3, 3 - at / T * 6, (at // 128 % 2) * 6.0 - 3])
    if buckets:
        p.table[1] = -math.inf
        p.table[2] = 4.0
        p.bias = bias_of(T, 4, p.bucket, 40, p.table, None, dev)
    p.Q[:, :] = 0
    p.K[:, :] = 0
    for h in range(4):
        p.Q[:, h * hd + h] = torch.where(at % 3 == 0, 1.0, torch.where(at % 3 == 1, -1.0, 0.05)).to(BF)
        p.K[:, h] = (along[h] * cap / p.scale).to(BF)
    return p


def many_equal(p, calls):
    f, b = check_forward(p)
    first = [x.clone() for x in (p.O, p.lse)]
    others = []
    for _ in range(calls):
        p.forward()
        others.append((p.O, p.lse))
    tda.tda_device_status()
    for O, lse in others:
        assert torch.equal(O, first[0]) and torch.equal(lse, first[1])
    return f, b


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("cap,buckets", [(30.0, 0), (30.0, 5), (57.0, 5), (62.3, 0), (80.0, 5)])
def test_capped_scores(dev, cap, buckets, hd):
    """Weights of a tile beyond 2^16 of the row's base, with and without the maximum first (a cap above 62.3)."""
    many_equal(at_the_cap(dev, cap, buckets, hd), 60)


@pytest.mark.parametrize("mask", ["causal", "full"])
@pytest.mark.parametrize("hd", [64, 128])
def test_slopes(dev, mask, hd):
    """Biases that fall with distance: nearer keys score higher, so that most tiles of keys raise the maximum by more than 2^8."""
    p = Problem(dev, 1, 2500, 6, 2, hd, BF, mask, slope=True)
    p.slope = torch.tensor([0.02, 0.06, 0.1, 0.2, 0.5, 1.0], device=dev)
    p.bias = bias_of(2500, 6, None, 0, None, p.slope, dev)
    f, b = many_equal(p, 60)
    check_backward(p, f, b)


def test_table_without_a_cap(dev):
    """A learned bias without a cap whose buckets step by more than 2^8 from tile to tile."""
    T = 1500
    p = Problem(dev, 1, T, 8, 2, 64, BF, "full", buckets=12, reach=T - 1)
    at = torch.arange(-(T - 1), T, device=dev)
    p.bucket = (at.abs() // 128).int()
    p.table = (torch.arange(12, device=dev)[:, None] * torch.linspace(-12, 12, 8, device=dev)).to(BF)
    p.bias = bias_of(T, 8, p.bucket, T - 1, p.table, None, dev)
    f, b = many_equal(p, 60)
    check_backward(p, f, b, grad=F32)
