"""Operators beside the token mixer, as a program built on the library calls them: linear attention with a
decay for each head (prompts, gradients, single tokens), the layer norm over channel groups that follows it,
and the router's balance loss with its gradients.

A case names its operator ("kind") and its sizes:
  attention  swimba_linear_attention: B prompts of L tokens
  gradient   swimba_linear_attention_backward: the gradients of queries, keys, values and entry states
  step       swimba_linear_attention_step: one token for each of B running sequences
  norm       swimba_layer_norm (and, with train, swimba_layer_norm_backward behind it)
  balance    swimba_balance_loss: loss, counts and the gradients of the router matrix and the token features
H heads read their queries and keys, [N] each, in G groups; a head's values have P entries.  A program keeps
the handle, the weights, the workspace and the output buffers from call to call; the inputs are new.
"""
import math
import random

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one chat turn: latency and launches
        dict(name="prefill_turn", kind="attention", dtype="bf16", B=1, L=93, H=16, G=16, N=64, P=64, state=True,
             packed=False),
        # prefill or training forward of a 2048-wide layer with 16 heads
        dict(name="prefill_mid", kind="attention", dtype="bf16", B=4, L=8192, H=16, G=16, N=128, P=128, state=False,
             packed=False),
        # one long document through a 1024-wide layer
        dict(name="prefill_long", kind="attention", dtype="bf16", B=1, L=65536, H=16, G=16, N=64, P=64, state=False,
             packed=False),
        # chunked prefill of a few ragged sequences on mixed streams: two groups of heads share keys and queries,
        # which lie side by side in one matrix
        dict(name="prefill_ragged", kind="attention", dtype="bf16", B=3, L=1531, H=36, G=2, N=128, P=64, state=True,
             packed=True),
        # one training step of the 2048-wide layer
        dict(name="gradient_mid", kind="gradient", dtype="bf16", B=4, L=8192, H=16, G=16, N=128, P=128, state=False,
             packed=False),
        # the fp32 path at the smallest workload: debugging, numerics references
        dict(name="gradient_tiny_fp32", kind="gradient", dtype="fp32", B=1, L=256, H=8, G=8, N=16, P=64, state=True,
             packed=False),
        # decoding: one user, and a full serving batch
        dict(name="step_one", kind="step", dtype="bf16", B=1, H=16, G=16, N=128, P=128, packed=False),
        dict(name="step_batch", kind="step", dtype="bf16", B=128, H=16, G=16, N=128, P=128, packed=False),
        # norms of a decode step's heads: latency
        dict(name="norm_token", kind="norm", dtype="bf16", rows=4, groups=16, width=128, train=False),
        # the norm of a training step, forward and backward
        dict(name="norm_train", kind="norm", dtype="bf16", rows=32768, groups=1, width=2048, train=True),
        # a short micro-batch through a router of four experts, padding behind every sequence
        dict(name="balance_short", kind="balance", dtype="bf16", B=2, L=187, F=768, E=4, k=1, du=True),
        # a training step's router
        dict(name="balance_mid", kind="balance", dtype="bf16", B=4, L=8192, F=2048, E=8, k=2, du=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["attention", "attention", "gradient", "gradient", "step", "norm", "norm", "balance", "balance"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if kind == "norm":
        groups = rng.choice([1, 1, 8, 16, 24])
        width = 8 * (_log_int(rng, 16, 320) if groups == 1 else rng.choice([4, 8, 12, 16]))
        top = 2.5e7 if dtype == "bf16" else 1.2e7
        return dict(kind=kind, dtype=dtype, rows=_log_int(rng, 1, top / (groups * width)), groups=groups, width=width,
                    train=rng.random() < 0.6)
    if kind == "balance":
        E = rng.choice([2, 4, 8, 8, 16, 32])
        F = 8 * _log_int(rng, 32, 256)
        tokens = _log_int(rng, 8, 16384 if dtype == "bf16" else 6000)
        B = min(rng.randint(1, 8), tokens)
        return dict(kind=kind, dtype=dtype, B=B, L=max(1, tokens // B), F=F, E=E, k=rng.randint(1, min(4, E - 1)),
                    du=rng.random() < 0.5)
    if dtype == "fp32":
        N, P = rng.choice([16, 32, 48, 64, 128]), rng.choice([32, 64, 80, 128])
    else:
        N, P = rng.choice([(64, 64), (64, 64), (128, 128), (128, 128), (128, 64), (64, 128), (32, 48), (96, 80)])
    G = rng.choice([1, 2, 4, 8, 12, 16])
    H = G * rng.choice([1, 1, 1, 2, 3])
    c = dict(kind=kind, dtype=dtype, H=H, G=G, N=N, P=P, packed=rng.random() < 0.3)
    if kind == "step":
        return dict(c, B=_log_int(rng, 1, 120))
    # tokens of the call over the logarithm, bounded by heads so that no drawn case outweighs the listed ones
    fast = dtype == "bf16" and N in (64, 128) and P in (64, 128)
    tokens = _log_int(rng, 30, (24000 if fast else 2500) * 16 // max(16, H))
    B = min(_log_int(rng, 1, 8), max(1, tokens // 20))
    return dict(c, B=B, L=max(1, tokens // B), state=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs

def _decays(H):
    """Slopes of a geometric family: the first head forgets within two tokens, the last after some hundred."""
    return torch.tensor([-(2.0 ** (-8.0 * (h + 1) / H)) for h in range(H)], device="cuda")


def _streams(case, n, gen, td):
    """Queries, keys [.., G, N] and values [.., H, P] of n leading dimensions."""
    G, N, H, P = case["G"], case["N"], case["H"], case["P"]
    if case["packed"]:                     # rows [keys | queries], as the mixed streams lie
        bc = torch.randn(*n, 2 * G * N, generator=gen, device="cuda").to(td)
        k, q = (t.unflatten(-1, (G, N)) for t in bc.split(G * N, dim=-1))
    else:
        q, k = (torch.randn(*n, G, N, generator=gen, device="cuda").to(td) for _ in range(2))
    return q, k, torch.randn(*n, H, P, generator=gen, device="cuda").to(td)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    td = _TYPES[case["dtype"]]
    s = dict(case=case)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)

    if case["kind"] in ("attention", "gradient", "step"):
        B, H, P, N = (case[n] for n in "BHPN")
        n = (B,) if case["kind"] == "step" else (B, case["L"])
        s["q"], s["k"], s["v"] = _streams(case, n, gen, td)
        s["log_decay"] = _decays(H)
        s["scale"] = N ** -0.5
        s["s0"] = normal(B, H, P, N, std=0.5) if case.get("state", True) else None
        if case["kind"] == "gradient":
            s["do"] = normal(B, case["L"], H, P, dtype=td)
            s["ds"] = normal(B, H, P, N, std=0.5) if case["state"] else None
    elif case["kind"] == "norm":
        rows, D = case["rows"], case["groups"] * case["width"]
        s["x"] = normal(rows, D, dtype=td) * 1.5 + 0.25
        s["w"], s["b"] = 1 + normal(D, std=0.1), normal(D, std=0.1)
        if case["train"]:
            s["dy"] = normal(rows, D, dtype=td)
    else:
        B, L, F, E, k = (case[n] for n in ("B", "L", "F", "E", "k"))
        T = B * L
        s["u"], s["W"] = normal(T, F, dtype=td), normal(E, F, std=0.02, dtype=td)
        lens = torch.randint((L + 1) // 2, L + 1, (B, 1), generator=gen, device="cuda")
        s["valid"] = (torch.arange(L, device="cuda") < lens).to(torch.uint8).reshape(T)
        logits = s["u"].float() @ s["W"].float().T       # the routing the layer's forward returned
        s["idx"] = logits.topk(k, dim=1).indices.to(torch.int32)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    from paper_2603_06938_b200 import binding as sb
    case = s["case"]
    dtype = sb.DTYPE_BF16 if case["dtype"] == "bf16" else sb.DTYPE_FP32
    td = _TYPES[case["dtype"]]
    s["sb"] = sb

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if case["kind"] in ("attention", "gradient", "step"):
        B, H, P, N, G = (case[n] for n in "BHPNG")
        h = s["h"] = sb.swimba_create(64, H, P, N, G, 1, 1, 128, dtype)
        if case["kind"] == "step":
            s["o"], s["s1"] = empty(B, H, P, dtype=td), empty(B, H, P, N)
        elif case["kind"] == "attention":
            L = case["L"]
            s["o"], s["s1"] = empty(B, L, H, P, dtype=td), empty(B, H, P, N)
            s["ws"] = empty(max(16, sb.swimba_linear_attention_workspace_bytes(h, B, L)), dtype=torch.uint8)
        else:
            L = case["L"]
            s["dq"], s["dk"] = empty(B, L, G, N, dtype=td), empty(B, L, G, N, dtype=td)
            s["dv"], s["ds0"] = empty(B, L, H, P, dtype=td), empty(B, H, P, N)
            s["ws"] = empty(max(16, sb.swimba_linear_attention_backward_workspace_bytes(h, B, L)), dtype=torch.uint8)
    elif case["kind"] == "norm":
        rows, groups, D = case["rows"], case["groups"], case["groups"] * case["width"]
        h = s["h"] = sb.swimba_create(64, 1, 16, 16, 1, 1, 1, 128, dtype)
        s["y"], s["mean"], s["rstd"] = empty(rows, D, dtype=td), empty(rows, groups), empty(rows, groups)
        if case["train"]:
            s["dx"], s["dw"], s["db"] = empty(rows, D, dtype=td), empty(D), empty(D)
            s["ws"] = empty(max(16, sb.swimba_layer_norm_workspace_bytes(h, rows, groups, case["width"])),
                            dtype=torch.uint8)
    else:
        F, E, k, T = case["F"], case["E"], case["k"], case["B"] * case["L"]
        h = s["h"] = sb.swimba_create(F, 1, 16, 16, 1, E, k, 128, dtype)
        s["weights"] = sb.make_weights(s["W"], None, None, None, None)
        s["loss"], s["counts"], s["mean"] = empty(1), empty(E, dtype=torch.int32), empty(E)
        s["dW"], s["du"] = empty(E, F), empty(T, F, dtype=td) if case["du"] else None
        s["ws"] = empty(max(16, sb.swimba_balance_loss_workspace_bytes(h, T)), dtype=torch.uint8)


# ---------------------------------------------------------------- the framework's calls

def _run_own(s):
    sb, case, h = s["sb"], s["case"], s["h"]
    kind = case["kind"]
    if kind == "attention":
        sb.swimba_linear_attention(h, s["log_decay"], s["q"], s["k"], s["v"], s["s0"], case["B"], case["L"], s["scale"],
                                   s["o"], s["s1"], s["ws"])
        return s["o"], s["s1"]
    if kind == "gradient":
        sb.swimba_linear_attention_backward(h, s["log_decay"], s["q"], s["k"], s["v"], s["s0"], s["do"], s["ds"],
                                            case["B"], case["L"], s["scale"], s["dq"], s["dk"], s["dv"], s["ds0"],
                                            s["ws"])
        return s["dq"], s["dk"], s["dv"], s["ds0"]
    if kind == "step":
        sb.swimba_linear_attention_step(h, s["log_decay"], s["q"], s["k"], s["v"], s["s0"], case["B"], s["scale"],
                                        s["o"], s["s1"])
        return s["o"], s["s1"]
    if kind == "norm":
        rows, groups, width = case["rows"], case["groups"], case["width"]
        sb.swimba_layer_norm(h, s["x"], s["w"], s["b"], rows, groups, width, 1e-5, s["y"], s["mean"], s["rstd"])
        if not case["train"]:
            return s["y"]
        sb.swimba_layer_norm_backward(h, s["dy"], s["x"], s["w"], s["mean"], s["rstd"], rows, groups, width, s["dx"],
                                      s["dw"], s["db"], s["ws"])
        return s["y"], s["dx"], s["dw"], s["db"]
    sb.swimba_balance_loss(h, s["weights"], s["u"], s["idx"], s["valid"], case["B"] * case["L"], 0.01, s["loss"],
                           s["counts"], s["mean"], s["dW"], s["du"], s["ws"])
    return (s["loss"], s["counts"], s["mean"], s["dW"]) + ((s["du"],) if case["du"] else ())


# ---------------------------------------------------------------- plain forms

def _heads(t, H):
    """[B, L, G, N] -> fp32 [B, H, L, N]: every head with the stream of its group."""
    return t.float().repeat_interleave(H // t.shape[2], dim=2).transpose(1, 2)


def _chunked(q, k, v, s0, g, scale, first=1, C=128):
    """o_t = scale S_t^T q_t with S_t = e^g S_{t-1} + k_t v_t^T, by chunks of C tokens; all fp32, [B, H, L, .].
    first: how often the decay has met the entry state at the first token (0: the decay follows the read)."""
    L = q.shape[2]
    S = s0
    i = torch.arange(C, device=q.device)
    dist = i[:, None] - i[None, :]
    g = g[:, None]
    mask = torch.where(dist >= 0, torch.exp(g[:, :, None] * dist.clamp(min=0)), 0.0)          # [H, C, C]
    into, out = [], []
    for t in range(0, L, C):
        qc, kc, vc = q[:, :, t:t + C], k[:, :, t:t + C], v[:, :, t:t + C]
        n = qc.shape[2]
        a = (qc @ kc.transpose(2, 3)) * mask[:, :n, :n]
        out.append((a @ vc + torch.exp(g * (i[:n] + first))[:, :, None] * (qc @ S)) * scale)
        S = torch.exp(g * n)[:, :, None] * S + (kc * torch.exp(g * (n - first - i[:n]))[:, :, None]).transpose(2, 3) @ vc
    return torch.cat(out, dim=2), S


def _plain_gradient(s):
    case = s["case"]
    B, H, P, N, G, L = (case[n] for n in "BHPNGL")
    td, g, sc = s["q"].dtype, s["log_decay"], s["scale"]
    q, k, v, do = (_heads(s[n], H) for n in ("q", "k", "v", "do"))
    zero = torch.zeros(B, H, P, N, device=q.device)
    s0 = s["s0"] if s["s0"] is not None else zero
    ds = s["ds"] if s["ds"] is not None else zero
    rev = lambda t: t.flip(2)
    dq, _ = _chunked(do, v, k, s0, g, sc)
    # R_t = e^g R_{t+1} + scale do_t q_t^T, entered by the final state's gradient (as it is at the last token)
    dk, r = _chunked(rev(v), rev(do * sc), rev(q), ds, g, 1.0, first=0)
    dv, _ = _chunked(rev(k), rev(q * sc), rev(do), ds.transpose(2, 3), g, 1.0, first=0)
    group = lambda t: t.transpose(1, 2).reshape(B, L, G, H // G, N).sum(3).to(td)
    return group(dq), group(rev(dk)), rev(dv).transpose(1, 2).to(td).contiguous(), r


def _plain_norm(s):
    case = s["case"]
    rows, groups, width = case["rows"], case["groups"], case["width"]
    x = s["x"].float().reshape(rows, groups, width)
    w, b = s["w"].reshape(groups, width), s["b"].reshape(groups, width)
    xc = x - x.mean(2, keepdim=True)
    rstd = torch.rsqrt((xc * xc).mean(2, keepdim=True) + 1e-5)
    xh = xc * rstd
    y = (xh * w + b).reshape(rows, -1).to(s["x"].dtype)
    if not case["train"]:
        return y
    dy = s["dy"].float().reshape(rows, groups, width)
    wd = dy * w
    dx = rstd * (wd - wd.mean(2, keepdim=True) - xh * (wd * xh).mean(2, keepdim=True))
    return y, dx.reshape(rows, -1).to(s["x"].dtype), (dy * xh).sum(0).reshape(-1), dy.sum(0).reshape(-1)


def _plain_balance(s):
    case = s["case"]
    E, k = case["E"], case["k"]
    u, W, valid = s["u"].float(), s["W"].float(), s["valid"].bool()
    g = u @ W.T
    p = torch.exp(g - g.max(1, keepdim=True).values)
    p = torch.where(valid[:, None], p / p.sum(1, keepdim=True), 0.0)
    hit = (s["idx"][:, :, None] == torch.arange(E, device=u.device)) & valid[:, None, None]
    counts = hit.sum((0, 1))
    n = valid.sum().double()
    f = counts.double() / (k * n)
    mean = (p.sum(0) / n.float())
    dev = (f - 1.0 / E).float()            # the shares lie close to 1 / E, and only what they differ by has a gradient
    dg = (0.01 * E / n).float() * p * (dev - (p * dev).sum(1, keepdim=True))
    out = (0.01 * E * (f.float() * mean).sum().reshape(1), counts.to(torch.int32), mean, dg.T @ u)
    return out + (((dg @ W).to(s["u"].dtype),) if case["du"] else ())


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "gradient":
        return _plain_gradient(s)
    if kind == "norm":
        return _plain_norm(s)
    if kind == "balance":
        return _plain_balance(s)
    H, g, sc = case["H"], s["log_decay"], s["scale"]
    if kind == "attention":
        q, k, v = (_heads(s[n], H) for n in "qkv")
        s0 = s["s0"].transpose(2, 3) if s["s0"] is not None else torch.zeros(
            case["B"], H, case["N"], case["P"], device=q.device)
        o, S = _chunked(q, k, v, s0, g, sc)
        return o.transpose(1, 2).to(s["q"].dtype).contiguous(), S.transpose(2, 3).contiguous()
    rep = H // case["G"]
    q, k = (s[n].float().repeat_interleave(rep, dim=1) for n in "qk")
    S = torch.exp(g)[:, None, None] * s["s0"] + s["v"].float()[:, :, :, None] * k[:, :, None, :]
    return (sc * (S * q[:, :, None, :]).sum(3)).to(s["q"].dtype), S


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- work

def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    kind = case["kind"]
    if kind == "norm":
        n = case["rows"] * case["groups"] * case["width"]
        par = 8 * case["groups"] * case["width"]
        return dict(bytes=(5 if case["train"] else 2) * n * e + (2 if case["train"] else 1) * par,
                    flops=(20 if case["train"] else 8) * n)
    if kind == "balance":
        T, F, E = case["B"] * case["L"], case["F"], case["E"]
        return dict(bytes=T * F * e * (2 if case["du"] else 1) + T * (4 * case["k"] + 1) + E * F * (e + 4),
                    flops=2 * T * F * E * (3 if case["du"] else 2))
    B, H, P, N, G = (case[n] for n in "BHPNG")
    T = B * case.get("L", 1)
    state = 4 * B * H * P * N
    if kind == "step":
        return dict(bytes=T * (2 * G * N + 2 * H * P) * e + 2 * state, flops=5 * T * H * P * N)
    if kind == "attention":
        # by chunks of 128 tokens: the causal half of two products inside the chunk, two with the state
        C = min(128, case["L"])
        return dict(bytes=T * (2 * G * N + 2 * H * P) * e + (2 if case["state"] else 1) * state,
                    flops=T * H * ((C + 1) * (N + P) + 4 * N * P))
    C = min(128, case["L"])
    return dict(bytes=T * (4 * G * N + 3 * H * P) * e + (3 if case["state"] else 1) * state,
                flops=T * H * (3 * (C + 1) * (N + P) + 10 * N * P))


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_scan(g, add_a, add_b, read, S, late=False):
    """Token by token: S <- e^g S + add_a_t add_b_t^T, yields S_t read_t; [L, B, H, .] streams, S [B, H, A, R].
    late: the decay follows the read of its token."""
    lam = torch.exp(g.double())[:, None, None]
    out = torch.empty(*add_a.shape, dtype=torch.float64, device=S.device)
    S = S.clone()
    for t in range(add_a.shape[0]):
        if not late:
            S.mul_(lam)
        S.addcmul_(add_a[t].unsqueeze(3), add_b[t].unsqueeze(2))
        torch.matmul(S, read[t].unsqueeze(3), out=out[t].unsqueeze(3))
        if late:
            S.mul_(lam)
    return out, S


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    kind = case["kind"]
    if kind == "norm":
        rows, groups, width = case["rows"], case["groups"], case["width"]
        if rows * groups * width > 10 ** 8:
            return None
        x = s["x"].double().view(rows, groups, width)
        w = s["w"].double().view(groups, width)
        var, mu = torch.var_mean(x, dim=2, keepdim=True, unbiased=False)
        sd = torch.sqrt(var + 1e-5)
        xh = (x - mu) / sd
        y = (xh * w + s["b"].double().view(groups, width)).view(rows, -1)
        if not case["train"]:
            return y
        dy = s["dy"].double().view(rows, groups, width)
        z = dy * w
        dx = (z - z.mean(2, True) - xh * (z * xh).mean(2, True)) / sd
        return y, dx.view(rows, -1), torch.einsum("rgw,rgw->gw", dy, xh).flatten(), dy.sum(0).flatten()
    if kind == "balance":
        E, k = case["E"], case["k"]
        ok = s["valid"].nonzero().flatten()
        u, W = s["u"].double()[ok], s["W"].double()
        p = torch.softmax(torch.einsum("tf,ef->te", u, W), dim=1)
        counts = torch.bincount(s["idx"][ok].flatten().long(), minlength=E)
        f = counts.double() / (k * len(ok))
        mean = p.mean(0)
        loss = 0.01 * E * torch.dot(f, mean)
        # of sum_t p_t . f / n through the softmax
        dg = (0.01 * E / len(ok)) * (p * f - p * (p @ f)[:, None])
        out = (loss.view(1), counts.to(torch.int32), mean, torch.einsum("te,tf->ef", dg, u))
        if not case["du"]:
            return out
        du = torch.zeros(s["u"].shape, dtype=torch.float64, device=u.device)
        du[ok] = torch.einsum("te,ef->tf", dg, W)
        return out + (du,)
    B, H, P, N, G = (case[n] for n in "BHPNG")
    if B * H * P * N * case.get("L", 1) > 3 * 10 ** 11:
        return None
    steps = kind == "step"

    def stream(name):                     # [L, B, H, .] in 64 bits, every head with its group's stream
        t = s[name].double()
        t = t.unsqueeze(1) if steps else t
        return t.repeat_interleave(H // t.shape[2], dim=2).transpose(0, 1).contiguous()

    q, k, v = stream("q"), stream("k"), stream("v")
    zero = torch.zeros(B, H, P, N, dtype=torch.float64, device=q.device)
    s0 = zero if s["s0"] is None else s["s0"].double()
    g, sc = s["log_decay"], s["scale"]
    if kind != "gradient":
        o, S = _exact_scan(g, v, k, q, s0)
        o = sc * o.transpose(0, 1)
        return (o[:, 0] if steps else o), S
    do = stream("do")
    ds = zero if s["ds"] is None else s["ds"].double()
    dq, _ = _exact_scan(g, k, v, do, s0.transpose(2, 3))
    dv, R = _exact_scan(g, do.flip(0) * sc, q.flip(0), k.flip(0), ds, late=True)
    dk, _ = _exact_scan(g, q.flip(0) * sc, do.flip(0), v.flip(0), ds.transpose(2, 3), late=True)
    heads = lambda t: t.transpose(0, 1).unflatten(2, (G, H // G)).sum(3)
    return (sc * heads(dq), heads(dk.flip(0)), dv.flip(0).transpose(0, 1), R)
