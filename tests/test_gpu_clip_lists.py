"""Gradient clipping of long lists: several launches' worth of tensors. Tolerances as in test_gpu_embedding_clip.py, 2^-24
per fp32 operation."""
import numpy as np
import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("count", [256, 257, 3000, 20000])
def test_long_lists(count):
    """The norm of all tensors, in the order of their list; every launch of the scaling reads one sum, which a single CTA
    made of all launches' partials (without that each of them would read all partials: quadratic in the list)."""
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    gen = torch.Generator(device="cuda").manual_seed(count)
    sizes = [1 + 13 * (i % 70) for i in range(count)]
    sizes[5] = 40000
    flat = torch.randn(sum(sizes), generator=gen, device="cuda")
    ts = list(flat.split(sizes))
    out = torch.full_like(flat, 9.0)
    refs = tda.tensor_list(ts, list(out.split(sizes)))
    wsb = tda.tda_grad_clip_workspace_size(refs, count)
    ws = torch.full((wsb,), 0x7F, dtype=torch.uint8, device="cuda")
    norm = torch.full((1,), 7.0, device="cuda")
    before = tda.tda_launch_count()
    tda.tda_grad_clip(refs, count, 2.0, norm, ws, wsb)
    launches = tda.tda_launch_count() - before
    tda.tda_device_status()
    want = float(flat.double().norm())
    assert abs(float(norm) - want) <= 20 * U * want
    ref = 2.0 / want * flat.double()
    assert bool(((out.double() - ref).abs() <= 24 * U * ref.abs()).all())
    again = torch.full((1,), 7.0, device="cuda")
    tda.tda_grad_clip(refs, count, 2.0, again, ws, wsb)
    assert torch.equal(norm, again)
    tables = -(-count // 256)
    assert launches == (2 if tables == 1 else 2 * tables + 1)
