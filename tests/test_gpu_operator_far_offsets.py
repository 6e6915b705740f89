"""The operators beside the mixer where element offsets pass 32 bits, and at the most sequences a call takes: strided rows of a
wide matrix against the same rows side by side, bit for bit; many short sequences against the definition."""
import pytest
import torch

import linear_attention_ref as ref
import test_gpu_balance_loss as bl
from test_gpu_layer_norm import handle as norm_handle
from paper_2603_06938_b200 import binding as sb

pytestmark = pytest.mark.gpu


def far(t, ld):
    """The rows of t [B, L, n, m] ld elements apart."""
    B, L, n, m = t.shape
    wide = torch.empty(B * L, ld, dtype=t.dtype, device="cuda")
    rows = wide[:, -n * m:]
    rows.copy_(t.reshape(B * L, n * m))
    return rows.view(B, L, n, m) if n * m == ld else rows.unflatten(0, (B, L)).unflatten(2, (n, m))


@pytest.mark.parametrize("dtype,N,P", [("bf16", 64, 64), ("bf16", 128, 128), ("bf16", 256, 32), ("fp32", 16, 64)])
def test_rows_far_apart(dtype, N, P):
    B, L, H = 2, 1400, 2
    ld = (2 ** 31 // (B * L) // 64 + 40) * 64                # the last rows start behind 2^31 elements
    i = ref.inputs(dtype, B, L, H, H, N, P, seed=3, grad=True, decays=[-0.01, -0.2])
    d = {n: t.cuda() for n, t in i.items() if torch.is_tensor(t)}
    h = ref.handle(i)
    ws = torch.empty(max(sb.swimba_linear_attention_workspace_bytes(h, B, L),
                         sb.swimba_linear_attention_backward_workspace_bytes(h, B, L)), dtype=torch.uint8, device="cuda")

    def run(q, k, v):
        o, s = torch.empty_like(d["v"]), torch.empty_like(d["s0"])
        sb.swimba_linear_attention(h, d["g"], q, k, v, d["s0"], B, L, i["scale"], o, s, ws)
        out = [torch.empty_like(d[n]) for n in ("q", "k", "v", "s0")]
        sb.swimba_linear_attention_backward(h, d["g"], q, k, v, d["s0"], d["do"], d["ds"], B, L, i["scale"], *out, ws)
        one, to = torch.empty_like(d["v"][:, 0]), torch.empty_like(d["s0"])
        sb.swimba_linear_attention_step(h, d["g"], q[:, L - 1], k[:, L - 1], v[:, L - 1], d["s0"], B, i["scale"], one, to)
        assert sb.swimba_status(h) == 0
        return o, s, *out, one, to

    want = run(d["q"], d["k"], d["v"])
    for n in ("q", "k", "v"):
        x = {m: d[m] for m in "qkv"}
        x[n] = far(d[n], ld)
        assert (B * L - 1) * ld > 2 ** 31
        assert all(torch.equal(a, b) for a, b in zip(run(**x), want)), n
        del x


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_norm_and_balance_of_far_rows(dtype):
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    rows, groups, width = 1100, 2, 96
    ld = (2 ** 31 // rows // 64 + 40) * 64
    h = norm_handle(dtype)
    x, dy = (torch.randn(rows, groups * width, device="cuda").to(td) for _ in range(2))
    ws = torch.empty(sb.swimba_layer_norm_workspace_bytes(h, rows, groups, width), dtype=torch.uint8, device="cuda")
    out = []
    for xx in (x, far(x.view(1, rows, 1, -1), ld).view(rows, -1)):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = (torch.empty(rows, groups, device="cuda") for _ in range(2))
        dw, db = (torch.empty(groups * width, device="cuda") for _ in range(2))
        sb.swimba_layer_norm(h, xx, None, None, rows, groups, width, 1e-5, y, mean, rstd)
        sb.swimba_layer_norm_backward(h, dy, xx, None, mean, rstd, rows, groups, width, dx, dw, db, ws)
        assert sb.swimba_status(h) == 0
        out.append((y, dx, mean, rstd, dw, db))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    del xx, out, x, dy
    # a router over tokens whose features pass 2^31 elements: the first and the last tokens' gradients by the definition
    F, E, k = 2048, 8, 2
    T = 2 ** 31 // F + 5000
    u = torch.empty(T, F, dtype=td, device="cuda")
    for a in range(0, T, 65536):
        u[a:a + 65536] = torch.randn(min(65536, T - a), F, device="cuda").to(td)
    W = (0.02 * torch.randn(E, F, device="cuda")).to(td)
    idx = torch.randint(0, E, (T, k), dtype=torch.int32, device="cuda")
    h = bl.handle(dtype, F, E, k)
    t, rc = bl.call(h, u, W, idx, None, T, F, E)
    assert rc == 0
    counts = torch.bincount(idx.flatten().long(), minlength=E)
    assert torch.equal(t["counts"].long(), counts)
    f = counts.double() / (k * T)
    for part in (slice(0, 500), slice(T - 500, T)):
        p = torch.softmax(u[part].double() @ W.double().T, dim=1)
        dg = bl.COEF * E / T * (p * (f - 1 / E) - p * (p @ (f - 1 / E))[:, None])
        mag = bl.COEF * E / T * (p * ((f - 1 / E).abs() + (p @ (f - 1 / E).abs())[:, None])) @ W.double().abs()
        want = dg @ W.double()
        # logits as in the other tests' bound, with |u||W| of these tokens
        n = 4 * F * 2.0 ** -24 * float((u[part].double().abs() @ W.double().abs().T).max()) + 2.0 ** -19
        err = (t["du"][part].double() - want).abs()
        assert bool((err <= bl.HALF[dtype] * want.abs() + (n + 2.0 ** -16) * mag + 1e-30).all())


@pytest.mark.parametrize("N,P", [(64, 64), (64, 128)])
def test_the_most_sequences(N, P):
    B, L, H = 65535, 2, 1
    i = ref.inputs("bf16", 1, 1, H, H, N, P, decays=[-0.3])
    h, g = ref.handle(i), i["g"].cuda()
    gen = torch.Generator("cuda").manual_seed(2)
    q, k = (torch.randn(B, L, H, N, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    v = torch.randn(B, L, H, P, generator=gen, device="cuda").to(torch.bfloat16)
    o, s = torch.empty_like(v), torch.empty(B, H, P, N, device="cuda")
    ws = torch.empty(sb.swimba_linear_attention_workspace_bytes(h, B, L), dtype=torch.uint8, device="cuda")
    sb.swimba_linear_attention(h, g, q, k, v, None, B, L, 1.0, o, s, ws)
    assert sb.swimba_status(h) == 0
    lam = float(torch.exp(g[0].double()))
    for a in range(0, B, 8192):
        x, y, z = (t[a:a + 8192, :, 0].double() for t in (q, k, v))
        own = (x * y).sum(2)
        other, m = (x[:, 1] * y[:, 0]).sum(1), lambda c, d: (c.abs() * d.abs()).sum(-1)
        w0 = own[:, :1] * z[:, 0]
        w1 = own[:, 1:] * z[:, 1] + lam * other[:, None] * z[:, 0]
        m0 = m(x[:, 0], y[:, 0])[:, None] * z[:, 0].abs()
        m1 = m(x[:, 1], y[:, 1])[:, None] * z[:, 1].abs() + lam * m(x[:, 1], y[:, 0])[:, None] * z[:, 0].abs()
        got = o[a:a + 8192, :, 0].double()
        slack = ref.slack("bf16", L)
        for gt, w, mm in ((got[:, 0], w0, m0), (got[:, 1], w1, m1)):
            assert bool(((gt - w).abs() <= 2.0 ** -8 * w.abs() + slack * mm).all())
        S = lam * z[:, 0, :, None] * y[:, 0, None, :] + z[:, 1, :, None] * y[:, 1, None, :]
        ms = lam * (z[:, 0, :, None] * y[:, 0, None, :]).abs() + (z[:, 1, :, None] * y[:, 1, None, :]).abs()
        assert bool(((s[a:a + 8192, 0].double() - S).abs() <= ref.slack("fp32", L) * ms).all())
