"""Layer norm of groups without variance: the mean is the value, what is normalised is zero to the bit, and so is its part of the
gradients, however large 1 / sqrt(eps) is.  (Values and widths whose sums are exact in 32 bits.)"""
import pytest
import torch

import helpers as hp
from test_gpu_layer_norm import TYPES, handle
from paper_2603_06938_b200 import binding as sb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [1e-5, 1e-12])
@pytest.mark.parametrize("value", [3.0, -1000.0, 0.0])
@pytest.mark.parametrize("groups,width", [(1, 768), (3, 40), (1, 1000), (2, 2056), (1, 4104), (16, 96), (1, 16384), (4, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_without_variance(dtype, groups, width, value, eps):
    rows, D, td = 9, groups * width, TYPES[dtype]
    gen = torch.Generator().manual_seed(width)
    x = torch.full((rows, D), value, dtype=td, device="cuda")
    # outputs' gradients whose sums over a group are exact: multiples of 1/8 up to 1
    dy = (torch.randint(-8, 9, (rows, D), generator=gen) / 8).to(td).cuda()
    b = torch.randn(D, generator=gen).cuda()
    h = handle(dtype)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty(rows, groups, device="cuda") for _ in range(2))
    dw, db = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    ws = torch.empty(sb.swimba_layer_norm_workspace_bytes(h, rows, groups, width), dtype=torch.uint8, device="cuda")
    sb.swimba_layer_norm(h, x, None, b, rows, groups, width, eps, y, mean, rstd)
    sb.swimba_layer_norm_backward(h, dy, x, None, mean, rstd, rows, groups, width, dx, dw, db, ws)
    assert sb.swimba_status(h) == 0
    assert bool((mean == x.view(rows, groups, width)[:, :, 0].float()).all())
    assert torch.equal(y, b.to(td).expand(rows, D))
    assert bool((dw == 0).all()), float(dw.abs().max())
    assert torch.equal(db, dy.float().sum(0))
    # dx = rstd (dy - mean(dy)): the mean, the difference and the product are rounded once each, the result to its type
    z = dy.double().cpu().view(rows, groups, width)
    r = rstd.double().cpu()[:, :, None]
    want = r * (z - z.mean(2, keepdim=True))
    half = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}[dtype]
    bound = half * want.abs() + 4 * 2.0 ** -24 * r * (z.abs() + z.mean(2, keepdim=True).abs())
    assert bool(((dx.double().cpu().view_as(want) - want).abs() <= bound).all())
    # 1 / sqrt(eps), eps rounded to 32 bits, to two ulps of the reciprocal root
    e = float(torch.tensor(eps, dtype=torch.float32))
    assert float((rstd.double() * e ** 0.5 - 1).abs().max()) <= 4 * 2.0 ** -23
