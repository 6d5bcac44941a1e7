"""Caps at either end of fp32's range: next to nothing of the scores is left, or nothing is taken from them."""
import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild
from test_gpu_attention import BF, F32, Problem, check_backward, check_forward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("buckets", [0, 6])
@pytest.mark.parametrize("cap", [1e-44, 1e-39, 2e-38, 1e-30, 1e-10])
def test_tiny_caps(dev, cap, buckets, dtype):
    """Scores are +-cap, but 0 where the product is 0: weights by the bias alone, and gradients only where the product is 0."""
    p = Problem(dev, 1, 200, 2, 1, 64, dtype, "causal", cap, buckets, 50 if buckets else 0)
    p.Q[::3] = 0
    p.K[::7] = 0
    p.cap = p.L.cap  # as fp32 holds it
    f, b = check_forward(p)
    check_backward(p, f, b)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("buckets", [0, 6])
@pytest.mark.parametrize("cap", [1.2e30, 1.3e30, 1e34, 5e36, 1e38, 2.5e38, 3.4e38])
def test_caps_beyond_the_scores(dev, cap, buckets, dtype):
    """Caps that bend nothing: the results and bounds of scores without a cap."""
    p = Problem(dev, 1, 200, 2, 1, 64, dtype, "causal", 0.0, buckets, 50 if buckets else 0)
    p.L.cap = cap
    f, b = check_forward(p)
    check_backward(p, f, b)
