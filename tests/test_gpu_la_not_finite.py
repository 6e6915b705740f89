"""Linear attention with infinities and NaN in the values of several tiles of one walk: outputs that see one are not finite,
all others keep the bits that they have without.  (An entry of V that is not finite reaches one column of the outputs: the
definition's row of the state, from its token on.)"""
import pytest
import torch

import helpers as hp
import linear_attention_ref as ref
from paper_2603_06938_b200 import binding as sb

pytestmark = pytest.mark.gpu

# heads that fill the SMs with one walk each, so that a sequence stays whole and a walk meets every tile
SHAPES = [(4, 37, 64, 64, 1500), (4, 37, 128, 64, 1300), (2, 74, 64, 128, 900), (4, 37, 128, 128, 1100)]


def spoil(t, tiles, L, seed):
    """In each of the given tiles an infinity or NaN at one place, another column for every tile; returns (copy, places)."""
    gen = torch.Generator().manual_seed(seed)
    t, at = t.clone(), []
    for n, tile in enumerate(tiles):
        for b in range(t.shape[0]):
            for h in range(t.shape[2]):
                tok = min(L - 1, tile * 128 + int(torch.randint(0, 128, (1,), generator=gen)))
                col = (7 * n + 3 * b) % t.shape[3]
                t[b, tok, h, col] = [float("inf"), float("nan"), -float("inf")][n % 3]
                at.append((b, tok, h, col))
    return t, at


def check(got, clean, at, after):
    """after: a place reaches the tokens behind it (else those in front), its own included."""
    bad = torch.zeros(got.shape, dtype=torch.bool)
    for b, tok, h, col in at:
        if after:
            bad[b, tok:, h, col] = True
        else:
            bad[b, :tok + 1, h, col] = True
    got, clean = got.cpu(), clean.cpu()
    assert torch.equal(got[~bad], clean[~bad])
    assert not torch.isfinite(got[bad]).any(), f"{int(torch.isfinite(got[bad]).sum())} of {int(bad.sum())} stay finite"


@pytest.mark.parametrize("tiles", [lambda n: range(n), lambda n: range(0, n, 2), lambda n: [1, 2], lambda n: [1, 3]],
                         ids=["all", "alternate", "neighbours", "two"])
@pytest.mark.parametrize("B,H,N,P,L", SHAPES)
def test_not_finite_in_several_tiles(B, H, N, P, L, tiles):
    i = ref.inputs("bf16", B, L, H, H, N, P, seed=L, decays=[-0.01, -0.001, -0.1], grad=True, state=False)
    tiles = list(tiles((L + 127) // 128))
    h = ref.handle(i)
    g = hp.dev(i["g"])
    ws = torch.empty(max(sb.swimba_linear_attention_workspace_bytes(h, B, L),
                         sb.swimba_linear_attention_backward_workspace_bytes(h, B, L)), dtype=torch.uint8, device="cuda")

    def forward(v):
        o = torch.empty(B, L, H, P, dtype=torch.bfloat16, device="cuda")
        sb.swimba_linear_attention(h, g, hp.dev(i["q"]), hp.dev(i["k"]), hp.dev(v), None, B, L, i["scale"], o, None, ws)
        return o

    def backward(**other):
        x = {n: hp.dev(other.get(n, i[n])) for n in ("q", "k", "v", "do")}
        out = [torch.empty(B, L, H, e, dtype=torch.bfloat16, device="cuda") for e in (N, N, P)]
        sb.swimba_linear_attention_backward(h, g, x["q"], x["k"], x["v"], None, x["do"], None, B, L, i["scale"], *out, None, ws)
        return out

    clean, grads = forward(i["v"]), backward()
    v, at = spoil(i["v"], tiles, L, 1)
    check(forward(v), clean, at, True)
    k, at = spoil(i["k"], tiles, L, 2)                   # dq takes keys as its values, walking forward
    check(backward(k=k)[0], grads[0], at, True)
    q, at = spoil(i["q"], tiles, L, 3)                   # dk queries, dv the outputs' gradients, both walking backward
    check(backward(q=q)[1], grads[1], at, False)
    do, at = spoil(i["do"], tiles, L, 4)
    check(backward(do=do)[2], grads[2], at, False)
    assert sb.swimba_status(h) == 0
