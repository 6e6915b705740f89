"""Linear attention with a decay for each head against the recurrence in 64 bits: prompts, gradients, single
tokens; sizes around tiles and segments, shared heads, strided rows, decays from none to total, states in place,
streams, captured calls, and tokens whose bits are infinities or NaN."""
import pytest
import torch

import helpers as hp
import linear_attention_ref as ref
from paper_2603_06938_b200 import binding as sb

pytestmark = pytest.mark.gpu


def put(i, packed):
    """Device tensors of the inputs; packed: keys and queries as columns of one matrix with a margin behind them."""
    d = {n: hp.dev(i.get(n)) for n in ("v", "s0", "g", "do", "ds")}
    B, L, G, N = i["B"], i["L"], i["G"], i["N"]
    if packed:
        m = torch.full((B * L, 2 * G * N + 32), float("nan"), dtype=i["q"].dtype, device="cuda")
        m[:, :G * N] = i["k"].reshape(B * L, G * N).cuda()
        m[:, G * N:2 * G * N] = i["q"].reshape(B * L, G * N).cuda()
        m = m.view(B, L, -1)
        d["k"], d["q"] = m[:, :, :G * N].unflatten(2, (G, N)), m[:, :, G * N:2 * G * N].unflatten(2, (G, N))
        w = torch.full((B * L, i["H"] * i["P"] + 64), float("nan"), dtype=i["v"].dtype, device="cuda")
        w[:, :i["H"] * i["P"]] = i["v"].reshape(B * L, -1).cuda()
        d["v"] = w.view(B, L, -1)[:, :, :i["H"] * i["P"]].unflatten(2, (i["H"], i["P"]))
    else:
        d["q"], d["k"] = hp.dev(i["q"]), hp.dev(i["k"])
    return d


def run_forward(i, packed=False, h=None):
    h = h or ref.handle(i)
    d = put(i, packed)
    o, ro = hp.with_canary((i["B"], i["L"], i["H"], i["P"]), i["v"].dtype, float("nan"))
    s, rs = hp.with_canary((i["B"], i["H"], i["P"], i["N"]), torch.float32, float("nan"))
    ws, rw = hp.with_canary((sb.swimba_linear_attention_workspace_bytes(h, i["B"], i["L"]),), torch.uint8, 0xff)
    sb.swimba_linear_attention(h, d["g"], d["q"], d["k"], d["v"], d["s0"], i["B"], i["L"], i["scale"], o, s, ws)
    assert sb.swimba_status(h) == 0, sb.swimba_last_error(h)
    assert hp.canary_intact(ro) and hp.canary_intact(rs) and hp.canary_intact(rw)
    return o, s


def run_backward(i, packed=False):
    h = ref.handle(i)
    d = put(i, packed)
    B, L, H, G, N, P = (i[n] for n in "BLHGNP")
    td = i["v"].dtype
    outs = [hp.with_canary(s, t, float("nan")) for s, t in
            (((B, L, G, N), td), ((B, L, G, N), td), ((B, L, H, P), td), ((B, H, P, N), torch.float32))]
    ws, rw = hp.with_canary((sb.swimba_linear_attention_backward_workspace_bytes(h, B, L),), torch.uint8, 0xff)
    sb.swimba_linear_attention_backward(h, d["g"], d["q"], d["k"], d["v"], d["s0"], d["do"], d["ds"], B, L, i["scale"],
                                        *(o for o, _ in outs), ws)
    assert sb.swimba_status(h) == 0, sb.swimba_last_error(h)
    assert all(hp.canary_intact(r) for _, r in outs) and hp.canary_intact(rw)
    return [o for o, _ in outs]


def check_forward(i, o, s):
    want, ws = ref.forward(i)
    mag, ms = ref.forward(i, absolute=True)
    ref.close(o, want, ref.slack(i["dtype"], i["L"]) * mag, i["dtype"], "o")
    ref.close(s, ws, ref.state_slack(i["dtype"], i["L"]) * ms, "fp32", "state")


def check_backward(i, got):
    want, mag = ref.backward(i), ref.backward(i, absolute=True)
    for n, g, w, m in zip(("dq", "dk", "dv"), got, want, mag):
        ref.close(g, w, ref.slack(i["dtype"], i["L"]) * m, i["dtype"], n)
    ref.close(got[3], want[3], ref.state_slack(i["dtype"], i["L"]) * mag[3], "fp32", "d state")


SHAPES = [  # dtype, H, G, N, P
    ("bf16", 7, 7, 128, 128), ("bf16", 7, 7, 64, 64), ("bf16", 6, 2, 128, 64), ("bf16", 7, 1, 64, 128),
    ("bf16", 4, 2, 32, 48), ("bf16", 3, 3, 96, 80), ("bf16", 2, 2, 256, 64), ("bf16", 2, 2, 16, 256),
    ("fp32", 8, 8, 16, 64), ("fp32", 6, 3, 48, 80), ("fp32", 7, 7, 128, 128), ("fp32", 2, 1, 256, 32),
]


@pytest.mark.parametrize("L", [1, 2, 63, 127, 128, 129, 300])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_at_tile_borders(shape, L):
    dtype, H, G, N, P = shape
    i = ref.inputs(dtype, 2, L, H, G, N, P, state=L % 2 == 1, seed=L)
    check_forward(i, *run_forward(i, packed=L % 3 == 0))


@pytest.mark.parametrize("L", [1, 2, 127, 128, 129, 300])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradients_at_tile_borders(shape, L):
    dtype, H, G, N, P = shape
    i = ref.inputs(dtype, 2, L, H, G, N, P, state=L % 2 == 1, seed=100 + L, grad=True)
    check_backward(i, run_backward(i, packed=L % 3 == 0))


@pytest.mark.parametrize("dtype,B,L,H,G,N,P", [("bf16", 1, 1531, 2, 2, 64, 64), ("bf16", 1, 2000, 1, 1, 128, 128),
                                               ("bf16", 3, 700, 2, 1, 128, 64), ("bf16", 1, 900, 1, 1, 48, 32),
                                               ("fp32", 1, 777, 1, 1, 32, 64)])
def test_sequences_cut_into_segments(dtype, B, L, H, G, N, P):
    i = ref.inputs(dtype, B, L, H, G, N, P, seed=7, decays=[-0.002, -0.03], grad=True)
    check_forward(i, *run_forward(i))
    check_backward(i, run_backward(i))


@pytest.mark.parametrize("B,H,G,N,L", [(5, 14, 14, 128, 1100), (10, 8, 4, 64, 700), (2, 37, 37, 128, 1536), (13, 12, 12, 128, 650)])
def test_walks_shared_between_blocks(B, H, G, N, L):
    """Heads of 128 values, as many as occupy a part of the SMs only: a walk's tiles are shared by several blocks, each of
    which carries the state through the tiles in front of its own.  (References on the GPU, in 64 bits.)"""
    i = ref.inputs("bf16", B, L, H, G, N, 128, seed=31)
    dev = {n: (t.cuda() if torch.is_tensor(t) else t) for n, t in i.items()}
    o, s = run_forward(i)
    zero = dev["s0"].double()
    q, k, v = (ref.per_head(dev[n], H) for n in ("q", "k", "v"))
    for f, bound in ((lambda x: x, False), (torch.abs, True)):
        w, ws = ref.scan(dev["g"], f(v), f(k), f(q), f(zero))
        if bound:
            mag, ms = i["scale"] * w.cpu(), ws.cpu()
        else:
            want, wants = i["scale"] * w.cpu(), ws.cpu()
    ref.close(o, want, ref.slack("bf16", L) * mag, "bf16", "o")
    ref.close(s, wants, ref.state_slack("bf16", L) * ms, "fp32", "state")


@pytest.mark.parametrize("B,H,G,N,L", [(1, 23, 23, 128, 1100), (4, 14, 7, 128, 640)])
def test_gradients_of_shared_walks(B, H, G, N, L):
    i = ref.inputs("bf16", B, L, H, G, N, 128, seed=33, grad=True)
    dev = {n: (t.cuda() if torch.is_tensor(t) else t) for n, t in i.items()}
    got = run_backward(i)
    want, mag = ref.backward(dev), ref.backward(dev, absolute=True)
    for n, g, w, m in zip(("dq", "dk", "dv"), got, want, mag):
        ref.close(g, w.cpu(), ref.slack("bf16", L) * m.cpu(), "bf16", n)
    ref.close(got[3], want[3].cpu(), ref.state_slack("bf16", L) * mag[3].cpu(), "fp32", "d state")


def test_gradients_agree_with_differences():
    """Central differences of sum(do * o) + sum(ds * S) in the fp32 path: outputs carry 2^-24 (L + ...) of their
    magnitudes, so a difference over a step of 1/8 (the map is linear in q, and bilinear in k, v: exact) is good to a
    thousandth of the largest gradient."""
    i = ref.inputs("fp32", 1, 40, 2, 1, 16, 32, seed=3, decays=[-0.05, -0.4], grad=True)
    got = run_backward(i)
    h = ref.handle(i)

    def loss(j):
        o, s = run_forward(j, h=h)
        return float((o.double().cpu() * j["do"].double()).sum() + (s.double().cpu() * j["ds"].double()).sum())
    gen = torch.Generator().manual_seed(1)
    for name, g in zip(("q", "k", "v", "s0"), got):
        for _ in range(6):
            at = tuple(int(torch.randint(0, n, (1,), generator=gen)) for n in i[name].shape)
            v = []
            for d in (0.125, -0.125):
                j = dict(i)
                j[name] = i[name].clone()
                j[name][at] += d
                v.append(loss(j))
            want = (v[0] - v[1]) / 0.25
            assert abs(float(g[at]) - want) <= 1e-3 * float(g.abs().max()), (name, at)


@pytest.mark.parametrize("dtype,H,G,N,P", [("bf16", 7, 7, 128, 128), ("bf16", 6, 2, 64, 64), ("bf16", 3, 3, 32, 48),
                                           ("fp32", 8, 2, 16, 64), ("fp32", 7, 7, 80, 40), ("bf16", 2, 2, 256, 64)])
@pytest.mark.parametrize("B", [1, 5, 33])
def test_steps_follow_a_prompt(dtype, H, G, N, P, B):
    """A prompt of 37 tokens in one call and four steps behind it, out of place and in place, against 41 tokens."""
    i = ref.inputs(dtype, B, 41, H, G, N, P, seed=11)
    d = put(i, packed=True)
    h = ref.handle(i)
    o = torch.full((B, 41, H, P), float("nan"), dtype=i["v"].dtype, device="cuda")
    head = torch.empty((B, 37, H, P), dtype=o.dtype, device="cuda")
    s = torch.empty((B, H, P, N), device="cuda")
    ws = torch.empty(sb.swimba_linear_attention_workspace_bytes(h, B, 37), dtype=torch.uint8, device="cuda")
    q, k, v = (d[n][:, :37].contiguous() for n in "qkv")
    sb.swimba_linear_attention(h, d["g"], q, k, v, d["s0"], B, 37, i["scale"], head, s, ws)
    o[:, :37] = head
    for t in range(37, 41):
        one = torch.empty((B, H, P), dtype=o.dtype, device="cuda")
        to = torch.full_like(s, float("nan")) if t % 2 else s
        sb.swimba_linear_attention_step(h, d["g"], d["q"][:, t], d["k"][:, t], d["v"][:, t], s, B, i["scale"], one, to)
        o[:, t], s = one, to
    assert sb.swimba_status(h) == 0
    check_forward(i, o, s)


@pytest.mark.parametrize("dtype,N,P", [("bf16", 128, 128), ("bf16", 64, 64), ("bf16", 32, 48), ("fp32", 32, 64)])
def test_state_in_place_and_pieces(dtype, N, P):
    """A prompt in three pieces that carry the state in one buffer, and a gradient call whose state's gradient goes
    back to where it came from."""
    i = ref.inputs(dtype, 1, 411, 3, 3, N, P, seed=5, grad=True, decays=[-0.01, 0.0, -0.3])
    d, h = put(i, False), ref.handle(i)
    o, s = torch.empty_like(d["v"]), d["s0"].clone()
    ws = torch.empty(sb.swimba_linear_attention_workspace_bytes(h, 1, 411), dtype=torch.uint8, device="cuda")
    for a, b in ((0, 200), (200, 201), (201, 411)):
        sb.swimba_linear_attention(h, d["g"], d["q"][:, a:b], d["k"][:, a:b], d["v"][:, a:b], s, 1, b - a, i["scale"],
                                   o[:, a:b], s, ws)
    check_forward(i, o, s)
    ds = d["ds"].clone()
    dq, dk, dv = torch.empty_like(d["q"]), torch.empty_like(d["k"]), torch.empty_like(d["v"])
    ws = torch.empty(sb.swimba_linear_attention_backward_workspace_bytes(h, 1, 411), dtype=torch.uint8, device="cuda")
    sb.swimba_linear_attention_backward(h, d["g"], d["q"], d["k"], d["v"], d["s0"], d["do"], ds, 1, 411, i["scale"], dq, dk,
                                        dv, ds, ws)
    check_backward(i, (dq, dk, dv, ds))
    assert sb.swimba_status(h) == 0


@pytest.mark.parametrize("dtype,N,P", [("bf16", 128, 128), ("bf16", 64, 64), ("bf16", 64, 128), ("bf16", 32, 48),
                                       ("fp32", 32, 64)])
@pytest.mark.parametrize("t", [0, 1, 63, 127, 128, 200, 290])
def test_no_token_sees_a_later_one(dtype, N, P, t):
    """Infinities and NaN in one token's row stay out of every token before it, of the other heads and of the other
    sequence; in the gradients, out of those that do not depend on it."""
    i = ref.inputs(dtype, 2, 291, 2, 2, N, P, seed=9, decays=[-0.02], grad=True)
    clean, cs = run_forward(i)
    grads = run_backward(i)
    for bad in (float("inf"), float("nan")):
        for name in ("q", "k", "v"):
            j = dict(i)
            j[name] = i[name].clone()
            j[name][0, t, 1] = bad
            o, s = run_forward(j)
            assert torch.equal(o[0, :t], clean[0, :t]) and torch.equal(o[1], clean[1])
            assert torch.equal(o[0, :, 0], clean[0, :, 0]) and torch.equal(s[1], cs[1])
            assert not torch.isfinite(o[0, t, 1]).any(), (bad, name)
            if name == "q":
                assert torch.equal(o[0, t + 1:], clean[0, t + 1:]) and torch.equal(s, cs)
            else:
                assert not torch.isfinite(s[0, 1]).all()
            g = run_backward(j)
            for a, b in zip(g[:3], grads[:3]):
                assert torch.equal(a[1], b[1]) and torch.equal(a[0, :, 0], b[0, :, 0])
            if name == "q":          # the gradient of a query does not depend on queries, those behind on this one
                assert torch.equal(g[0], grads[0])
                assert torch.equal(g[1][0, t + 1:], grads[1][0, t + 1:]) and torch.equal(g[2][0, t + 1:], grads[2][0, t + 1:])
            else:
                assert torch.equal(g[0][0, :t], grads[0][0, :t])
        j = dict(i)
        j["do"] = i["do"].clone()
        j["do"][0, t, 1] = bad
        g = run_backward(j)
        assert torch.equal(g[1][0, t + 1:], grads[1][0, t + 1:]) and torch.equal(g[2][0, t + 1:], grads[2][0, t + 1:])
        assert torch.equal(g[0][0, :t], grads[0][0, :t]) and torch.equal(g[0][0, t + 1:], grads[0][0, t + 1:])


@pytest.mark.parametrize("dtype,B,H,N,P,L", [("bf16", 5, 14, 128, 128, 700), ("bf16", 1, 2, 64, 64, 1900), ("fp32", 1, 2, 32, 64, 900),
                                             ("bf16", 2, 100, 128, 128, 300)])
def test_states_in_place_where_blocks_share_a_walk(dtype, B, H, N, P, L):
    """States that go back to where they came from, when several blocks read what one of them writes in the end: the bits of
    separate buffers, eagerly and replayed."""
    i = ref.inputs(dtype, B, L, H, H, N, P, seed=41, grad=True, decays=[-0.001, -0.02])
    want_o, want_s = run_forward(i)
    want_g = run_backward(i)
    d, h = put(i, False), ref.handle(i)
    o, s, ds = torch.empty_like(d["v"]), d["s0"].clone(), d["ds"].clone()
    dq, dk, dv = torch.empty_like(d["q"]), torch.empty_like(d["k"]), torch.empty_like(d["v"])
    ws = torch.empty(sb.swimba_linear_attention_workspace_bytes(h, B, L), dtype=torch.uint8, device="cuda")
    wb = torch.empty(sb.swimba_linear_attention_backward_workspace_bytes(h, B, L), dtype=torch.uint8, device="cuda")

    def call():
        sb.swimba_linear_attention(h, d["g"], d["q"], d["k"], d["v"], s, B, L, i["scale"], o, s, ws)
        sb.swimba_linear_attention_backward(h, d["g"], d["q"], d["k"], d["v"], d["s0"], d["do"], ds, B, L, i["scale"], dq, dk,
                                            dv, ds, wb)

    def same():
        torch.cuda.synchronize()
        assert torch.equal(o, want_o) and torch.equal(s, want_s)
        assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv, ds), want_g))
        s.copy_(d["s0"])
        ds.copy_(d["ds"])
        for t in (o, dq, dk, dv):
            t.fill_(float("nan"))

    call()
    same()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        graph.replay()
        same()
    assert sb.swimba_status(h) == 0


@pytest.mark.parametrize("L", [5, 300, 1100])
@pytest.mark.parametrize("N,P", [(16, 8), (112, 72), (48, 120), (128, 8), (80, 64), (16, 128)])
def test_heads_between_the_tiles_sizes(N, P, L):
    """Head sizes that tiles of 64 or 128 entries hold with a margin: states, shared heads and strided rows of the head's
    own size, and nothing of the head beside it."""
    i = ref.inputs("bf16", 2, L, 4, 2, N, P, seed=N + P + L, decays=[-0.002, -0.03], grad=True, state=L != 300)
    check_forward(i, *run_forward(i, packed=L == 1100))
    check_backward(i, run_backward(i, packed=L == 1100))


@pytest.mark.parametrize("t", [0, 63, 128, 290])
@pytest.mark.parametrize("N,P", [(96, 80), (112, 40), (16, 72)])
def test_no_token_sees_a_later_one_between_the_tiles_sizes(N, P, t):
    test_no_token_sees_a_later_one("bf16", N, P, t)


@pytest.mark.parametrize("dtype,N,P", [("bf16", 128, 128), ("bf16", 48, 64), ("fp32", 64, 64)])
def test_captured_replayed_and_on_two_streams(dtype, N, P):
    i = ref.inputs(dtype, 1, 500, 2, 2, N, P, seed=21, grad=True, decays=[-0.01])
    want_o, want_s = run_forward(i)
    want_g = run_backward(i)
    jobs = []
    for _ in range(2):                       # each its own handle, buffers and stream
        d, h = put(i, False), ref.handle(i)
        x = dict(d=d, h=h, st=torch.cuda.Stream(), o=torch.empty_like(d["v"]), s=torch.empty_like(d["s0"]),
                 g=[torch.empty_like(t) for t in want_g],
                 ws=torch.empty(sb.swimba_linear_attention_workspace_bytes(h, 1, 500), dtype=torch.uint8, device="cuda"),
                 wb=torch.empty(sb.swimba_linear_attention_backward_workspace_bytes(h, 1, 500), dtype=torch.uint8,
                                device="cuda"))
        jobs.append(x)

    def call(x, stream=None):
        d = x["d"]
        sb.swimba_linear_attention(x["h"], d["g"], d["q"], d["k"], d["v"], d["s0"], 1, 500, i["scale"], x["o"], x["s"],
                                   x["ws"], stream)
        sb.swimba_linear_attention_backward(x["h"], d["g"], d["q"], d["k"], d["v"], d["s0"], d["do"], d["ds"], 1, 500,
                                            i["scale"], *x["g"], x["wb"], stream)
    torch.cuda.synchronize()
    for _ in range(3):
        for x in jobs:
            call(x, x["st"])
    torch.cuda.synchronize()
    for x in jobs:
        assert torch.equal(x["o"], want_o) and torch.equal(x["s"], want_s)
        assert all(torch.equal(a, b) for a, b in zip(x["g"], want_g))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(jobs[0])
    for t in (jobs[0]["o"], jobs[0]["s"], *jobs[0]["g"]):
        t.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(jobs[0]["o"], want_o) and all(torch.equal(a, b) for a, b in zip(jobs[0]["g"], want_g))


def test_many_sequences_and_empty_calls():
    i = ref.inputs("bf16", 40, 3, 2, 1, 64, 64, seed=2)
    check_forward(i, *run_forward(i))
    h = ref.handle(i)
    t = torch.full((16,), 7.0, device="cuda")
    assert sb.lib().swimba_linear_attention(h.ptr, None, None, 0, None, 0, None, 0, None, 0, 5, 1.0, None, None, None, 0,
                                            None) == 0
    assert sb.swimba_status(h) == 0 and bool((t == 7).all())
