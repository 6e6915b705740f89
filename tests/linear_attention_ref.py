"""Linear attention with a decay for each head, token by token in 64 bits, with the sums of magnitudes that bound
what roundings can do (test plumbing; shares nothing with the library)."""
from __future__ import annotations

import torch

from paper_2603_06938_b200 import binding as sb

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}         # largest relative error of one rounding


def scan(g, add_a, add_b, read, S, late=False):
    """S <- e^g S + a_t b_t^T per token, out_t = S read_t; streams [B, L, H, .], S [B, H, A, R], 64 bits.
    late: the decay follows the read of its token.  Returns out [B, L, H, A] and the last state."""
    lam = torch.exp(g.double())[:, None, None]
    S, out = S.clone(), []
    for t in range(add_a.shape[1]):
        if not late:
            S = lam * S
        S = S + add_a[:, t, :, :, None] * add_b[:, t, :, None, :]
        out.append((S * read[:, t, :, None, :]).sum(-1))
        if late:
            S = lam * S
    return torch.stack(out, 1), S


def per_head(t, H):
    return t.double().repeat_interleave(H // t.shape[2], dim=2)


def forward(i, absolute=False):
    """(o, S) of the inputs i, or the same sums over magnitudes."""
    f = torch.abs if absolute else (lambda x: x)
    q, k, v = (f(per_head(i[n], i["H"])) for n in ("q", "k", "v"))
    s0 = f(i["s0"].double()) if i["s0"] is not None else torch.zeros(i["B"], i["H"], i["P"], i["N"], dtype=torch.float64, device=q.device)
    o, S = scan(i["g"], v, k, q, s0)
    return i["scale"] * o, S


def backward(i, absolute=False):
    f = torch.abs if absolute else (lambda x: x)
    H, G, sc, g = i["H"], i["G"], i["scale"], i["g"]
    q, k, v, do = (f(per_head(i[n], H)) for n in ("q", "k", "v", "do"))
    zero = torch.zeros(i["B"], H, i["P"], i["N"], dtype=torch.float64, device=q.device)
    s0 = f(i["s0"].double()) if i["s0"] is not None else zero
    ds = f(i["ds"].double()) if i["ds"] is not None else zero
    dq, _ = scan(g, k, v, do, s0.transpose(2, 3))
    dv, R = scan(g, do.flip(1) * sc, q.flip(1), k.flip(1), ds, late=True)
    dk, _ = scan(g, q.flip(1) * sc, do.flip(1), v.flip(1), ds.transpose(2, 3), late=True)
    group = lambda t: t.unflatten(2, (G, H // G)).sum(3)
    return group(sc * dq), group(dk.flip(1)), dv.flip(1), R


def inputs(dtype, B, L, H, G, N, P, state=True, seed=0, decays=None, grad=False):
    gen = torch.Generator().manual_seed(seed)
    td = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    r = lambda *s: torch.randn(*s, generator=gen)
    i = dict(dtype=dtype, B=B, L=L, H=H, G=G, N=N, P=P, scale=N ** -0.5)
    i["q"], i["k"], i["v"] = r(B, L, G, N).to(td), r(B, L, G, N).to(td), r(B, L, H, P).to(td)
    # from no decay at all to one that leaves nothing behind
    i["g"] = torch.tensor([decays[h % len(decays)] for h in range(H)] if decays else
                          [[0.0, -0.004, -0.06, -0.5, -3.0, -60.0, -float("inf")][h % 7] for h in range(H)])
    i["s0"] = 0.5 * r(B, H, P, N) if state else None
    if grad:
        i["do"] = r(B, L, H, P).to(td)
        i["ds"] = 0.5 * r(B, H, P, N) if state else None
    return i


def handle(i, flags=0):
    return sb.swimba_create(64, i["H"], i["P"], i["N"], i["G"], 1, 1, 128,
                            sb.DTYPE_BF16 if i["dtype"] == "bf16" else sb.DTYPE_FP32, flags)


def close(got, want, bound, dtype, what):
    """|got - want| <= half a step of the stored type + bound, element by element."""
    got = got.double().cpu()
    err = (got - want).abs() - HALF[dtype] * want.abs() - bound
    assert bool((err <= 0).all()), f"{what}: worst excess {float(err.max()):.3e} of {float(want.abs().max()):.3e}"
    assert torch.isfinite(got).all(), what


def slack(dtype, L):
    """Relative to the sum of magnitudes.  bf16: scores and carried state are rounded to bf16 once each as operands of
    the next product (2^-8 either; a term passes one of them), fp32 sums of L + 512 terms and decay factors whose
    exponents are rounded (2^-24 a term or power; exponents up to 150 in log2, 2^-17) beside that."""
    fp32 = (L + 512) * 2.0 ** -24 + 2.0 ** -16
    return fp32 + (2.0 ** -8 if dtype == "bf16" else 0.0)


def state_slack(dtype, L):
    """States are fp32: what they add is taken in two bf16 parts, 2^-16 of a term."""
    return slack("fp32", L) + (2.0 ** -16 if dtype == "bf16" else 0.0)
