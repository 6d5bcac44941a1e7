"""The norm's outputs in the place of its inputs, where the header allows it: the bits of a call with outputs of their own."""
import pytest
import torch

import paper_2609_38767_gb300 as tda
from paper_2609_38767_gb300 import build as tbuild
from test_gpu_norm import CASES, EPS, KIND

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    tbuild.build()
    tda.load()
    return torch.device("cuda:0")


def rows(M, d, dtype, gen, dev):
    return torch.randn((M, d), generator=gen, device=dev).to(dtype)


MANY = [(M, d) for M, d, _, _ in CASES] + [(4000, 256), (3000, 1024), (2500, 4096)]  # several rows a group: the next one on its way


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,d", MANY)
def test_gradient_in_place(dev, M, d, dtype):
    """dx is dy, or dres."""
    gen = torch.Generator(device=dev).manual_seed(M + 7 * d)
    h, dy, dres = (rows(M, d, dtype, gen, dev) for _ in range(3))
    w = rows(1, d, dtype, gen, dev).view(d)
    rstd = torch.rsqrt(h.float().square().mean(1) + EPS)
    wsb = tda.tda_rmsnorm_workspace_size(M, d)
    ws = torch.empty(wsb, dtype=torch.uint8, device=dev)

    def call(dy, dres, dx):
        dw = torch.full((d,), 7.0, device=dev)
        tda.tda_rmsnorm_backward(KIND[dtype], h, d, rstd, w, dy, d, dres, d, M, d, dx, d, dw, tda.TDA_F32, 0.0, ws, wsb)
        tda.tda_device_status()
        return dw

    for res in (None, dres):
        dx = torch.full_like(h, 7.0)
        dw = call(dy, res, dx)
        assert torch.isfinite(dx.float()).all()
        mine = dy.clone()
        assert torch.equal(call(mine, res, mine), dw) and torch.equal(mine, dx)
    mine = dres.clone()
    assert torch.equal(call(dy, mine, mine), dw) and torch.equal(mine, dx)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,d", MANY)
def test_norm_in_place(dev, M, d, dtype):
    """h and y in the place of x and r."""
    gen = torch.Generator(device=dev).manual_seed(M + 9 * d)
    x, r = (rows(M, d, dtype, gen, dev) for _ in range(2))
    w = rows(1, d, dtype, gen, dev).view(d)

    def call(x, r, h, y):
        rstd = torch.full((M,), 7.0, device=dev)
        tda.tda_rmsnorm_forward(KIND[dtype], x, d, r, d, M, d, w, EPS, h, d, y, d, rstd)
        tda.tda_device_status()
        return rstd

    h, y = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    rstd = call(x, r, h, y)
    for into in ("x", "r", "xr", "rx", ".x", ".r"):  # of h and of y, "." a tensor of its own
        a, b = x.clone(), r.clone()
        at = {"x": a, "r": b, ".": torch.full_like(x, 7.0)}
        mine_h, mine_y = at[into[0]], at[into[1]] if len(into) > 1 else torch.full_like(x, 7.0)
        assert torch.equal(call(a, b, mine_h, mine_y), rstd) and torch.equal(mine_h, h) and torch.equal(mine_y, y), into
