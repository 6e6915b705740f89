"""The router's balance loss, its counts and gradients against the definition in 64 bits."""
import pytest
import torch

import helpers as hp
from paper_2603_06938_b200 import binding as sb
from paper_2603_06938_b200 import synth

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
COEF = 0.01


def reference(u, W, idx, valid, E, k):
    ok = valid.bool()
    u, W = u.double(), W.double()
    n = int(ok.sum())
    um = torch.where(ok[:, None], u, 0.0)
    p = torch.where(ok[:, None], torch.softmax(um @ W.T, dim=1), 0.0)
    e = idx[ok].flatten().long()
    counts = torch.bincount(e[(e >= 0) & (e < E)], minlength=E)
    if n == 0:
        z = torch.zeros
        return dict(loss=0.0, counts=counts, mean=z(E).double(), dW=z(E, u.shape[1]).double(), du=z(u.shape).double(),
                    dW_mag=z(E, u.shape[1]).double(), du_mag=z(u.shape).double(), logit=0.0)
    f, mean = counts.double() / (k * n), p.sum(0) / n
    d = f - 1.0 / E
    dg = COEF * E / n * (p * d - p * (p @ d)[:, None])
    # what a relative error of p makes of dg
    dg_mag = COEF * E / n * (p * (d.abs() + (p @ d.abs())[:, None]))
    return dict(loss=COEF * E * float(f @ mean), counts=counts, mean=mean, dW=dg.T @ um, du=dg @ W,
                dW_mag=dg_mag.T @ um.abs(), du_mag=dg_mag @ W.abs(), logit=float((um.abs() @ W.abs().T).max()))


def handle(dtype, F, E, k, flags=0):
    return sb.swimba_create(F, 1, 16, 16, 1, E, k, 128, sb.DTYPE_BF16 if dtype == "bf16" else sb.DTYPE_FP32, flags)


def make(dtype, T, F, E, k, seed, std=0.05):
    gen = torch.Generator().manual_seed(seed)
    u, W = torch.randn(T, F, generator=gen).to(TYPES[dtype]), (std * torch.randn(E, F, generator=gen)).to(TYPES[dtype])
    idx = (u.float() @ W.float().T).topk(k, dim=1).indices.to(torch.int32)
    return u, W, idx, (torch.rand(T, generator=gen) < 0.8).to(torch.uint8)


def call(h, u, W, idx, valid, T, F, E, want_dW=True, want_du=True, dW=None):
    w = sb.make_weights(W, None, None, None, None)
    o = {n: hp.with_canary(s, t, fill) for n, s, t, fill in
         (("loss", (1,), torch.float32, float("nan")), ("counts", (E,), torch.int32, -1),
          ("mean", (E,), torch.float32, float("nan")), ("du", (T, F), u.dtype, float("nan")),
          ("dW", (E, F), torch.float32, float("nan")))}
    if dW is not None:
        o["dW"][0].copy_(dW)
    ws, raw = hp.with_canary((sb.swimba_balance_loss_workspace_bytes(h, T),), torch.uint8, 0xff)
    t = {n: x for n, (x, _) in o.items()}
    sb.swimba_balance_loss(h, w, u, idx, valid, T, COEF, t["loss"], t["counts"], t["mean"], t["dW"] if want_dW else None,
                           t["du"] if want_du else None, ws, accumulate=dW is not None)
    rc = sb.swimba_status(h)
    assert all(hp.canary_intact(r) for _, r in o.values()) and hp.canary_intact(raw)
    return t, rc


def check(t, r, dtype, T, F, E):
    # logits: F products in fp32, so a probability is off by 2 F 2^-24 of the largest |u||W| (and exp's ulps)
    p = 2 * F * 2.0 ** -24 * r["logit"] + 2.0 ** -20
    n = (T + F + 64) * 2.0 ** -24 + 2 * p
    assert torch.equal(t["counts"].cpu().long(), r["counts"])
    assert bool(((t["mean"].double().cpu() - r["mean"]).abs() <= n * r["mean"] + 1e-30).all())
    assert abs(float(t["loss"]) - r["loss"]) <= n * abs(r["loss"])
    assert bool(((t["dW"].double().cpu() - r["dW"]).abs() <= n * r["dW_mag"] + 1e-30).all())
    # (dg may pass through 16-bit halves on its way into a product: 2^-16 of it)
    assert bool(((t["du"].double().cpu() - r["du"]).abs() <= HALF[dtype] * r["du"].abs() + (n + 2.0 ** -16) * r["du_mag"] + 1e-30).all())


CASES = [("bf16", 1, 64, 4, 1), ("bf16", 15, 768, 4, 1), ("bf16", 374, 768, 4, 2), ("bf16", 1000, 2048, 8, 2),
         ("bf16", 33, 200, 16, 4), ("bf16", 129, 72, 64, 8), ("bf16", 5000, 512, 2, 1), ("bf16", 64, 1024, 16, 2),
         ("bf16", 700, 2056, 8, 3), ("bf16", 257, 4096, 8, 2), ("bf16", 600, 256, 33, 3), ("bf16", 2100, 1536, 32, 2),
         ("fp32", 1, 8, 2, 1), ("fp32", 300, 256, 4, 2), ("fp32", 77, 1000, 64, 2), ("fp32", 1025, 512, 8, 1)]


@pytest.mark.parametrize("dtype,T,F,E,k", CASES)
def test_against_the_definition(dtype, T, F, E, k):
    u, W, idx, valid = make(dtype, T, F, E, k, seed=T)
    ud = u.clone()
    ud[valid == 0] = float("nan")             # padding may hold anything
    h = handle(dtype, F, E, k)
    ud, Wd, di, dv = ud.cuda(), W.cuda(), idx.cuda(), valid.cuda()
    t, rc = call(h, ud, Wd, di, dv, T, F, E)
    assert rc == 0
    r = reference(u, W, idx, valid, E, k)
    check(t, r, dtype, T, F, E)
    assert bool((t["du"][valid.cuda() == 0] == 0).all())
    again, _ = call(h, ud, Wd, di, dv, T, F, E)
    assert all(torch.equal(t[n], again[n]) for n in t)
    only, _ = call(h, ud, Wd, di, dv, T, F, E, want_dW=False, want_du=False)
    assert torch.equal(only["loss"], t["loss"]) and torch.equal(only["mean"], t["mean"])
    part, _ = call(h, ud, Wd, di, dv, T, F, E, want_du=False)
    assert torch.equal(part["dW"], t["dW"]) and bool(part["du"].isnan().all())
    part, _ = call(h, ud, Wd, di, dv, T, F, E, want_dW=False)
    assert torch.equal(part["du"], t["du"]) and bool(part["dW"].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_mask_no_valid_token_and_one_expert(dtype):
    u, W, idx, _ = make(dtype, 90, 128, 4, 2, seed=1)
    h = handle(dtype, 128, 4, 2)
    t, rc = call(h, u.cuda(), W.cuda(), idx.cuda(), None, 90, 128, 4)
    assert rc == 0
    check(t, reference(u, W, idx, torch.ones(90), 4, 2), dtype, 90, 128, 4)
    t, rc = call(h, u.cuda(), W.cuda(), idx.cuda(), torch.zeros(90, dtype=torch.uint8, device="cuda"), 90, 128, 4)
    assert rc == 0
    check(t, reference(u, W, idx, torch.zeros(90), 4, 2), dtype, 90, 128, 4)
    one = handle(dtype, 128, 1, 1)
    t, rc = call(one, u.cuda(), W[:1].cuda().contiguous(), torch.zeros(90, 1, dtype=torch.int32, device="cuda"), None, 90, 128, 1)
    assert rc == 0 and abs(float(t["loss"]) - COEF) < 1e-8 and bool((t["dW"] == 0).all()) and bool((t["du"] == 0).all())


def test_indices_outside_the_experts():
    u, W, idx, valid = make("bf16", 50, 64, 4, 2, seed=3)
    idx[3, 0], idx[9, 1], idx[11, 0] = 4, -1, 2 ** 30
    valid[:] = 1
    for flags, want in ((0, 0), (1, sb.ERR_DEVICE_BOUNDS)):
        h = handle("bf16", 64, 4, 2, flags)
        t, rc = call(h, u.cuda(), W.cuda(), idx.cuda(), valid.cuda(), 50, 64, 4)
        assert rc == want
        assert torch.equal(t["counts"].cpu().long(), reference(u, W, idx, valid, 4, 2)["counts"])


def test_unaligned_mask_capture_and_accumulation():
    u, W, idx, valid = make("bf16", 333, 256, 8, 2, seed=8)
    h = handle("bf16", 256, 8, 2)
    u, W, idx = u.cuda(), W.cuda(), idx.cuda()
    mask = torch.zeros(340, dtype=torch.uint8, device="cuda")[3:336]
    mask.copy_(valid)
    want, _ = call(h, u, W, idx, valid.cuda(), 333, 256, 8)
    got, _ = call(h, u, W, idx, mask, 333, 256, 8)
    assert all(torch.equal(want[n], got[n]) for n in want)
    base = torch.randn(8, 256, device="cuda") * float(want["dW"].abs().max())
    got, _ = call(h, u, W, idx, mask, 333, 256, 8, dW=base)
    # one more rounding than the sum of the two
    assert bool(((got["dW"] - (base + want["dW"])).abs() <= (333 + 8) * 2.0 ** -24 * (base.abs() + want["dW"].abs()) +
                 400 * 2.0 ** -24 * want["dW"].abs().max()).all())
    w = sb.make_weights(W, None, None, None, None)
    t = {n: torch.empty_like(x) for n, x in want.items()}
    ws = torch.empty(sb.swimba_balance_loss_workspace_bytes(h, 333), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sb.swimba_balance_loss(h, w, u, idx, mask, 333, COEF, t["loss"], t["counts"], t["mean"], t["dW"], t["du"], ws)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(want[n], t[n]) for n in want)


def test_routed_linear_attention_trains_a_router():
    """The operators as a layer uses them: mixed streams from the router, linear attention over their keys and queries,
    a norm per head; back through norm and attention; the balance loss added to the router's gradient.  Against the
    same in 64 bits from the library's own mixed streams."""
    import linear_attention_ref as ref
    B, L, F, H, P, N, E, k = 2, 160, 128, 4, 64, 64, 4, 2
    T = B * L
    cfg = synth.LayerConfig("routed", "bf16", B, L, F, H, P, N, H, E, k, 128)
    inp = synth.make_inputs(cfg, seed=70)
    h = hp.create_handle(cfg)
    w, keep = hp.device_weights(inp)
    u = hp.dev(inp["u"]).view(T, F)
    x = hp.dev(inp["x"])
    S = 2 * H * N
    BC = torch.empty(T, S, dtype=torch.bfloat16, device="cuda")
    idx, wt = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")
    ws = torch.empty(max(sb.swimba_workspace_bytes(h, B, L), sb.swimba_linear_attention_backward_workspace_bytes(h, B, L),
                         sb.swimba_linear_attention_workspace_bytes(h, B, L), sb.swimba_balance_loss_workspace_bytes(h, T),
                         sb.swimba_layer_norm_workspace_bytes(h, T, H, P)), dtype=torch.uint8, device="cuda")
    sb.swimba_route_mix(h, w, u, T, BC, idx, wt, ws)
    kk, qq = (t.unflatten(2, (H, N)) for t in BC.view(B, L, S).split(H * N, dim=2))
    g = torch.tensor([-0.5, -0.1, -0.02, 0.0], device="cuda")
    nw, nb = torch.ones(H * P, device="cuda"), torch.zeros(H * P, device="cuda")
    o, y, dx = (torch.empty_like(x) for _ in range(3))
    mean, rstd = torch.empty(T, H, device="cuda"), torch.empty(T, H, device="cuda")
    dy = torch.randn(B, L, H, P, device="cuda").to(torch.bfloat16)
    dw, db = torch.empty(H * P, device="cuda"), torch.empty(H * P, device="cuda")
    dq, dk = (torch.empty(B, L, H, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dv = torch.empty_like(x)
    sb.swimba_linear_attention(h, g, qq, kk, x, None, B, L, N ** -0.5, o, None, ws)
    sb.swimba_layer_norm(h, o.view(T, -1), nw, nb, T, H, P, EPS := 1e-5, y.view(T, -1), mean, rstd)
    sb.swimba_layer_norm_backward(h, dy.view(T, -1), o.view(T, -1), nw, mean, rstd, T, H, P, dx.view(T, -1), dw, db, ws)
    sb.swimba_linear_attention_backward(h, g, qq, kk, x, None, dx, None, B, L, N ** -0.5, dq, dk, dv, None, ws)
    loss, counts = torch.empty(1, device="cuda"), torch.empty(E, dtype=torch.int32, device="cuda")
    dW = torch.zeros(E, F, device="cuda")
    sb.swimba_balance_loss(h, w, u, idx, None, T, COEF, loss, counts, None, dW, None, ws, accumulate=True)
    assert sb.swimba_status(h) == 0
    i = dict(dtype="bf16", B=B, L=L, H=H, G=H, N=N, P=P, scale=N ** -0.5, g=g.cpu(), q=qq.cpu(), k=kk.cpu(), v=x.cpu(),
             s0=None, ds=None, do=dx.cpu())
    want, mag = ref.forward(i)[0], ref.forward(i, absolute=True)[0]
    ref.close(o, want, ref.slack("bf16", L) * mag, "bf16", "o")
    od = o.cpu().double()
    xh = (od - od.mean(3, keepdim=True)) / torch.sqrt(od.var(3, keepdim=True, unbiased=False) + EPS)
    assert bool(((y.double().cpu() - xh).abs() <= 2.0 ** -8 * xh.abs() + 1e-4).all())
    for n, got, a, m in zip(("dq", "dk", "dv"), (dq, dk, dv), ref.backward(i), ref.backward(i, absolute=True)):
        ref.close(got, a, ref.slack("bf16", L) * m, "bf16", n)
    r = reference(u.cpu(), inp["W_r"], idx.cpu(), torch.ones(T), E, k)
    assert torch.equal(counts.cpu().long(), r["counts"]) and abs(float(loss) - r["loss"]) <= 1e-4 * r["loss"]
    assert bool(((dW.double().cpu() - r["dW"]).abs() <= 1e-3 * r["dW_mag"]).all())
