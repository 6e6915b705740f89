"""Exit states of linear attention where heads remember thousands of tokens: sums of positive terms, whose errors nothing hides,
against the definition in 64 bits, within what 32-bit sums that round can do."""
import pytest
import torch

from paper_2603_06938_b200 import binding as sb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def state(g, k, v, s0=None):
    """sum_t lambda^(L - 1 - t) v_t k_t^T + lambda^L s0 in 64 bits; k, v [B, L, H, .]."""
    L, g = k.shape[1], g.double()
    S = 0.0 if s0 is None else s0.double()
    for t in range(0, L, 1024):
        kc, vc = (x[:, t:t + 1024].double().transpose(1, 2) for x in (k, v))
        n = kc.shape[2]
        w = torch.exp(g[:, None] * torch.arange(n - 1, -1, -1, device=k.device).double())
        S = torch.exp(g * n)[:, None, None] * S + (vc * w[:, :, None]).transpose(2, 3) @ kc
    return S


def handle(H, N, P):
    return sb.swimba_create(64, H, P, N, H, 1, 1, 128, sb.DTYPE_BF16)


def workspace(h, B, L):
    n = max(sb.swimba_linear_attention_workspace_bytes(h, B, L), sb.swimba_linear_attention_backward_workspace_bytes(h, B, L))
    return torch.empty(n, dtype=torch.uint8, device="cuda")


# Relative errors of a sum of positive terms, the running sum of T tiles being t / T of the result at tile t (less, with a decay):
#   inside a tile     24 additions of the tensor cores at most, each of which may cut 2^-23 off
#   from tile to tile two roundings of the running sum: T / 2 times 2^-23
#   a term's weight   exp2f (2 ulps) of a product of rounded factors, times two others, then three bf16 parts: 2^-20 in all
# Sequences cut into segments (the last case: nine, of 57 tiles) add up half of that many tiles in the pieces, then all tiles of
# the last segment onto the whole state, one rounding each.
def bound(tiles):
    return 24 * 2 * U + tiles * U + 2.0 ** -20


CASES = [(4, 8192, 16, 128, 128, 64), (2, 8192, 74, 128, 128, 64), (1, 8192, 16, 64, 128, 64), (1, 16384, 1, 128, 128, 128),
         (4, 8192, 37, 64, 64, 64), (1, 8192, 16, 128, 64, 64), (1, 65536, 16, 64, 64, 100)]


@pytest.mark.parametrize("g", [0.0, -2.3e-5, -2.0 ** -12])
@pytest.mark.parametrize("B,L,H,N,P,tiles", CASES)
def test_states_of_slow_heads(B, L, H, N, P, tiles, g):
    gen = torch.Generator("cuda").manual_seed(L + H)
    q, k = (torch.randn(B, L, H, N, generator=gen, device="cuda").abs().to(torch.bfloat16) for _ in range(2))
    v, do = (torch.randn(B, L, H, P, generator=gen, device="cuda").abs().to(torch.bfloat16) for _ in range(2))
    decay = torch.full((H,), g, device="cuda")
    h = handle(H, N, P)
    ws = workspace(h, B, L)
    o, s = torch.empty_like(v), torch.empty(B, H, P, N, device="cuda")
    sb.swimba_linear_attention(h, decay, q, k, v, None, B, L, 1.0, o, s, ws)
    assert sb.swimba_status(h) == 0
    want = state(decay, k, v)
    worst = float(((s.double() - want).abs() / want).max())
    assert worst <= bound(tiles), f"state: {worst:.2e} of {bound(tiles):.2e}"
    dq, dk, dv, ds = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(s)
    sb.swimba_linear_attention_backward(h, decay, q, k, v, None, do, None, B, L, 1.0, dq, dk, dv, ds, ws)
    assert sb.swimba_status(h) == 0
    want = torch.exp(decay.double())[:, None, None] * state(decay, q.flip(1), do.flip(1))
    worst = float(((ds.double() - want).abs() / want).max())
    assert worst <= bound(tiles), f"d state: {worst:.2e} of {bound(tiles):.2e}"


@pytest.mark.parametrize("B,L,H,N,P", [(4, 16384, 37, 64, 64), (4, 16384, 37, 128, 128), (1, 65536, 2, 64, 64), (1, 65536, 3, 128, 128)])
def test_the_decay_itself(B, L, H, N, P):
    """A state that nothing is added to decays by lambda a token: over many entries the roundings of its products cancel, and
    what is left is the error of the factor, multiplied up.  (128 tiles, each off by half of 2^-24 the same way: 2^-18.)"""
    z = torch.zeros(B, L, H, max(N, P), dtype=torch.bfloat16, device="cuda")
    assert N == P
    s0 = 1 + torch.rand(B, H, P, N, generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    decay = torch.full((H,), -2.3e-5, device="cuda")
    h = handle(H, N, P)
    ws = workspace(h, B, L)
    o, s = torch.empty_like(z), torch.empty_like(s0)
    sb.swimba_linear_attention(h, decay, z, z, z, s0, B, L, 1.0, o, s, ws)
    assert sb.swimba_status(h) == 0
    # (the decay's exponent is rounded to 32 bits once: as many parts in 2^24 as lambda^L has e-folds)
    want = torch.exp(decay.double() * L)[:, None, None] * s0.double()
    mean = float(((s.double() - want) / want).mean())
    assert abs(mean) <= U * (1 + 2.3e-5 * L), f"{mean:.2e}"


@pytest.mark.parametrize("t", [0, 37, 100, 126])
@pytest.mark.parametrize("N,P", [(64, 64), (128, 64), (64, 128), (128, 128), (48, 80)])
def test_one_term(N, P, t):
    """A state that one token of a tile adds to is one product, weight times value times key.  Of it 18 parts in 2^24: the
    weight's exponent, rounded twice, of less than 1 (1), exp2f twice (8), two products (2), three bf16 parts (1) and as
    many additions that cut (6).  Two bf16 parts would leave up to 2^-17, 128 parts."""
    B, L, H = 2, 128, 4
    gen = torch.Generator("cuda").manual_seed(t)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)
    q, k, v, do = (torch.zeros(B, L, H, n, dtype=torch.bfloat16, device="cuda") for n in (N, N, P, P))
    for x in (q, k, v, do):
        x[:, t] = r(*x[:, t].shape)
    decay = torch.tensor([-0.004, -0.003, -0.002, -0.001], device="cuda")
    scale = 0.37
    h = handle(H, N, P)
    ws = workspace(h, B, L)
    o, s, ds = torch.empty_like(v), torch.empty(B, H, P, N, device="cuda"), torch.empty(B, H, P, N, device="cuda")
    sb.swimba_linear_attention(h, decay, q, k, v, None, B, L, scale, o, s, ws)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    sb.swimba_linear_attention_backward(h, decay, q, k, v, None, do, None, B, L, scale, dq, dk, dv, ds, ws)
    assert sb.swimba_status(h) == 0
    lam = torch.exp(decay.double())[:, None, None]
    one = lambda a, b: a[:, t, :, :, None].double() * b[:, t, :, None, :].double()
    f32 = float(torch.tensor(scale))
    for got, want in ((s, lam ** (L - 1 - t) * one(v, k)), (ds, f32 * lam ** (t + 1) * one(do, q))):
        assert bool(((got.double() - want).abs() <= 18 * U * want.abs()).all()), float(((got.double() - want) / want).abs().max())
