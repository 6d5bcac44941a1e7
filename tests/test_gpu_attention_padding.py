"""Batches with examples, and long ends of examples, that are padding: items without keys in any number between others, for the tensor
cores and the CUDA cores, with results, zeros in the padding and equal bits from equal calls."""
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


def pad(p, lengths):
    """Example n has lengths[n] tokens, the rest is padding; what lies there is not a number."""
    doc = torch.where(torch.arange(p.T)[None] < torch.tensor(lengths)[:, None], 0, -1).int().to(p.dev)
    p.range = torch.empty((p.N, p.T, 2), dtype=torch.int32, device=p.dev)
    tda.tda_attention_ranges(p.N, p.T, doc, None, True, 0, p.range)
    at = torch.arange(p.T, device=p.dev)
    p.seen = (at >= p.range[..., :1]) & (at < p.range[..., 1:])
    gone = (doc < 0).reshape(-1)
    p.Q[gone], p.K[gone], p.V[gone], p.dO[gone] = (float("nan"),) * 4


SCORES = [(0.0, 0, 0, False), (30.0, 12, 40, False), (0.0, 0, 0, True)]
LENGTHS = {
    "every other": lambda N, T, g: [T if n % 2 else 0 for n in range(N)],
    "one in five": lambda N, T, g: [T if n % 5 == 2 else 0 for n in range(N)],
    "the last only": lambda N, T, g: [T if n == N - 1 else 0 for n in range(N)],
    "the first only": lambda N, T, g: [T if n == 0 else 0 for n in range(N)],
    "any": lambda N, T, g: [max(0, int(torch.randint(-T, T + 1, (1,), generator=g))) for n in range(N)],
    "none": lambda N, T, g: [0] * N,
}


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cap,buckets,reach,slope", SCORES)
@pytest.mark.parametrize("which", list(LENGTHS))
@pytest.mark.parametrize("N,T,H,KV,hd", [(150, 5, 16, 4, 64), (60, 130, 16, 8, 128), (40, 70, 9, 3, 64)])
def test_padded_examples(dev, N, T, H, KV, hd, which, cap, buckets, reach, slope, dtype):
    p = Problem(dev, N, T, H, KV, hd, dtype, "full", cap, buckets, reach, slope)
    pad(p, LENGTHS[which](N, T, torch.Generator().manual_seed(N)))
    f, b = check_forward(p)
    check_backward(p, f, b, grad=F32)
    gone = ~p.seen.any(2).reshape(-1)
    assert all((x[gone] == 0).all() for x in (p.O, p.dQ, p.dK, p.dV))
    first = [x.clone() for x in (p.O, p.lse, p.dQ, p.dK, p.dV)]
    for _ in range(5):
        p.forward()
        p.backward(grad=F32)
        tda.tda_device_status()
        assert all(torch.equal(x, y) for x, y in zip(first, (p.O, p.lse, p.dQ, p.dK, p.dV)))


@pytest.mark.parametrize("cap,buckets,reach,slope", SCORES)
@pytest.mark.parametrize("lengths", [[3000, 100], [90, 2900], [1500, 1501], [3000, 0], [1, 3000]])
def test_long_padding(dev, lengths, cap, buckets, reach, slope):
    p = Problem(dev, 2, 3000, 8, 2, 64, BF, "full", cap, buckets, reach, slope)
    pad(p, lengths)
    f, b = check_forward(p)
    check_backward(p, f, b, grad=F32)
