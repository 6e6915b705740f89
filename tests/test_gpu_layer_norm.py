"""Layer norm over channel groups and its gradients against the definition in 64 bits."""
import pytest
import torch

import helpers as hp
from paper_2603_06938_b200 import binding as sb

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-5


def handle(dtype):
    return sb.swimba_create(64, 1, 16, 16, 1, 1, 1, 128, sb.DTYPE_BF16 if dtype == "bf16" else sb.DTYPE_FP32)


def reference(x, dy, w, b, rows, groups, width):
    x, dy = x.double().view(rows, groups, width), dy.double().view(rows, groups, width)
    w = torch.ones(groups, width, dtype=torch.float64) if w is None else w.double().view(groups, width)
    b = torch.zeros(groups, width, dtype=torch.float64) if b is None else b.double().view(groups, width)
    mu = x.mean(2, keepdim=True)
    rs = 1 / torch.sqrt(((x - mu) ** 2).mean(2, keepdim=True) + EPS)
    xh, z = (x - mu) * rs, dy * w
    m0, m1 = z.mean(2, keepdim=True), (z * xh).mean(2, keepdim=True)
    return dict(y=xh * w + b, dx=rs * (z - m0 - xh * m1), dw=(dy * xh).sum(0), db=dy.sum(0), mu=mu[..., 0], rs=rs[..., 0],
                # magnitudes that roundings act on: x / sigma of a term, the sums of z
                my=(x.abs() + mu.abs()) * rs * w.abs() + b.abs(),
                mx=rs * (z.abs() + z.abs().mean(2, keepdim=True) + (xh.abs() + 1) * (z * xh).abs().mean(2, keepdim=True)
                         + (x.abs() + mu.abs()) * rs * (m1.abs() + z.abs().mean(2, keepdim=True))),
                mw=(dy.abs() * ((x.abs() + mu.abs()) * rs)).sum(0), mb=dy.abs().sum(0))


def run(dtype, rows, groups, width, weights=True, seed=0, margin=0, offset=0.0):
    gen = torch.Generator().manual_seed(seed)
    td, D = TYPES[dtype], groups * width
    x = (1.5 * torch.randn(rows, D, generator=gen) + offset).to(td)
    dy = torch.randn(rows, D, generator=gen).to(td)
    w = 1 + 0.1 * torch.randn(D, generator=gen) if weights else None
    b = 0.1 * torch.randn(D, generator=gen) if weights else None
    h = handle(dtype)
    wide = torch.full((rows, D + margin), float("nan"), dtype=td, device="cuda")
    wide[:, :D] = x.cuda()
    xd = wide[:, :D]
    outs = {n: hp.with_canary(s, t, float("nan")) for n, s, t in
            (("y", (rows, D), td), ("dx", (rows, D), td), ("mean", (rows, groups), torch.float32),
             ("rstd", (rows, groups), torch.float32), ("dw", (D,), torch.float32), ("db", (D,), torch.float32))}
    o = {n: t for n, (t, _) in outs.items()}
    ws, raw = hp.with_canary((sb.swimba_layer_norm_workspace_bytes(h, rows, groups, width),), torch.uint8, 0xff)
    sb.swimba_layer_norm(h, xd, hp.dev(w), hp.dev(b), rows, groups, width, EPS, o["y"], o["mean"], o["rstd"])
    sb.swimba_layer_norm_backward(h, hp.dev(dy), xd, hp.dev(w), o["mean"], o["rstd"], rows, groups, width, o["dx"], o["dw"],
                                  o["db"], ws)
    assert sb.swimba_status(h) == 0
    assert all(hp.canary_intact(r) for _, r in outs.values()) and hp.canary_intact(raw)
    r = reference(x, dy, w, b, rows, groups, width)
    # fp32 inside: statistics of `width` terms and sums over `rows`, each term to 2^-24 and a few operations
    n = (width + 32) * 2.0 ** -24
    for name, want, mag, k in (("y", r["y"], r["my"], n), ("dx", r["dx"], r["mx"], 4 * n)):
        err = (o[name].double().cpu().view_as(want) - want).abs()
        assert bool((err <= HALF[dtype] * want.abs() + k * mag).all()), name
    for name, want, mag in (("dw", r["dw"], r["mw"]), ("db", r["db"], r["mb"])):
        err = (o[name].double().cpu().view_as(want) - want).abs()
        assert bool((err <= (rows + width + 64) * 2.0 ** -24 * mag).all()), name
    return o, (h, xd, dy, w, b, ws)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,groups,width", [(1, 1, 8), (1, 1, 2048), (3, 1, 1000), (17, 1, 768), (9, 1, 4104),
                                               (5, 1, 16384), (70, 16, 64), (1, 16, 128), (33, 24, 96), (301, 3, 40),
                                               (2, 64, 256), (5, 300, 8), (2000, 2, 24), (1, 7, 2056), (4001, 1, 64)])
def test_norm_and_gradients(dtype, rows, groups, width):
    run(dtype, rows, groups, width, seed=rows)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,groups,width", [(50, 8, 2048), (7, 5, 1032), (900, 3, 4096), (3, 2, 16384), (40, 9, 776), (700, 1, 2056)])
def test_wide_groups(dtype, rows, groups, width):
    """Groups of several places a thread: some of them, or one, to a block."""
    run(dtype, rows, groups, width, seed=rows)
    run(dtype, rows, groups, width, weights=False, margin=8)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_without_weights_strided_rows_and_a_large_mean(dtype):
    run(dtype, 77, 2, 128, weights=False, margin=64)
    run(dtype, 40, 1, 512, margin=8, offset=100.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_constant_rows(dtype):
    """A row without variance: y is the bias, to the bit."""
    h = handle(dtype)
    x = torch.full((5, 256), 3.0, dtype=TYPES[dtype], device="cuda")
    b = torch.arange(256, device="cuda").float()
    y = torch.empty_like(x)
    sb.swimba_layer_norm(h, x, None, b, 5, 1, 256, EPS, y, None, None)
    assert torch.equal(y, b.to(x.dtype).expand(5, 256))


def test_rows_do_not_touch_each_other_and_results_repeat():
    o, (h, xd, dy, w, b, ws) = run("bf16", 300, 4, 64, seed=4)
    x2 = xd.clone()
    x2[7, 64:128] = float("nan")
    y = torch.empty_like(o["y"])
    sb.swimba_layer_norm(h, x2, hp.dev(w), hp.dev(b), 300, 4, 64, EPS, y, None, None)
    bad = torch.zeros(300, 256, dtype=torch.bool, device="cuda")
    bad[7, 64:128] = True
    assert torch.equal(y[~bad], o["y"][~bad]) and torch.isnan(y[bad]).all()
    for _ in range(3):
        dw, db, dx = torch.empty_like(o["dw"]), torch.empty_like(o["db"]), torch.empty_like(o["dx"])
        sb.swimba_layer_norm_backward(h, hp.dev(dy), xd, hp.dev(w), o["mean"], o["rstd"], 300, 4, 64, dx, dw, db, ws)
        assert torch.equal(dw, o["dw"]) and torch.equal(db, o["db"]) and torch.equal(dx, o["dx"])
        dx.fill_(0)
        sb.swimba_layer_norm_backward(h, hp.dev(dy), xd, hp.dev(w), o["mean"], o["rstd"], 300, 4, 64, dx, None, None, None)
        assert torch.equal(dx, o["dx"])


def test_no_rows_clear_the_weight_gradients():
    h = handle("bf16")
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    m = torch.empty(0, 1, device="cuda")
    dw, db = torch.full((64,), 5.0, device="cuda"), torch.full((64,), 5.0, device="cuda")
    sb.swimba_layer_norm(h, e, None, None, 0, 1, 64, EPS, e, m, m)
    sb.swimba_layer_norm_backward(h, e, e, None, m, m, 0, 1, 64, e, dw, db, None)
    torch.cuda.synchronize()
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_captured_and_replayed():
    o, (h, xd, dy, w, b, ws) = run("bf16", 100, 2, 64, seed=6)
    dyd, wd, bd = hp.dev(dy), hp.dev(w), hp.dev(b)
    out = {n: torch.full_like(t, float("nan")) for n, t in o.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sb.swimba_layer_norm(h, xd, wd, bd, 100, 2, 64, EPS, out["y"], out["mean"], out["rstd"])
        sb.swimba_layer_norm_backward(h, dyd, xd, wd, out["mean"], out["rstd"], 100, 2, 64, out["dx"], out["dw"], out["db"], ws)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[n], o[n]) for n in o)
