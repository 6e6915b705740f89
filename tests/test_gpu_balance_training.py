"""The balance loss at the sizes of a training step: counts in a launch of their own (more than 8192 entries of the active
sets), several tiles of tokens a block, up to 16 experts on the tensor cores; masks that leave out single tokens, whole tiles and
the end; gradients of the features wanted or not."""
import pytest
import torch

import test_gpu_balance_loss as bl
from paper_2603_06938_b200 import binding as sb

pytestmark = pytest.mark.gpu

CASES = [(9000, 256, 8, 2), (8200, 64, 8, 1), (30001, 128, 3, 1), (12005, 512, 16, 1), (5000, 2048, 16, 4), (7003, 1008, 9, 3),
         (6000, 2048, 8, 2)]


def masks(T, gen):
    """Tokens that count: most of them; two sequences in three padded by halves (whole tiles); all but the last tile."""
    some = (torch.rand(T, generator=gen) < 0.8).to(torch.uint8)
    half = ((torch.arange(T) // 500 % 3 == 0) | (torch.arange(T) % 500 < 250)).to(torch.uint8)
    front = (torch.arange(T) < T // 16 * 16 - 16).to(torch.uint8)
    return {"some": some, "half": half, "front": front, "all": torch.ones(T, dtype=torch.uint8)}


@pytest.mark.parametrize("which", ["some", "half", "front", "all"])
@pytest.mark.parametrize("T,F,E,k", CASES)
def test_against_the_definition(T, F, E, k, which):
    u, W, idx, _ = bl.make("bf16", T, F, E, k, seed=T + E, std=0.02)
    valid = masks(T, torch.Generator().manual_seed(T))[which]
    ud = u.clone()
    ud[valid == 0] = float("nan")             # padding may hold anything
    h = bl.handle("bf16", F, E, k)
    ud, Wd, di, dv = ud.cuda(), W.cuda(), idx.cuda(), (None if which == "all" else valid.cuda())
    t, rc = bl.call(h, ud, Wd, di, dv, T, F, E)
    assert rc == 0
    bl.check(t, bl.reference(u, W, idx, valid, E, k), "bf16", T, F, E)
    assert bool((t["du"][valid.cuda() == 0] == 0).all())
    for _ in range(5):
        part, rc = bl.call(h, ud, Wd, di, dv, T, F, E, want_du=False)
        assert rc == 0 and all(torch.equal(part[n], t[n]) for n in ("loss", "counts", "mean", "dW"))
        again, rc = bl.call(h, ud, Wd, di, dv, T, F, E)
        assert rc == 0 and all(torch.equal(again[n], t[n]) for n in t)
    part, rc = bl.call(h, ud, Wd, di, dv, T, F, E, want_dW=False)
    assert rc == 0 and torch.equal(part["du"], t["du"]) and torch.equal(part["loss"], t["loss"])


@pytest.mark.parametrize("flags,want", [(0, 0), (1, sb.ERR_DEVICE_BOUNDS)])
def test_indices_outside_the_experts(flags, want):
    T, F, E, k = 9000, 256, 16, 1
    u, W, idx, _ = bl.make("bf16", T, F, E, k, seed=5)
    idx[3, 0], idx[8999, 0], idx[4000, 0] = E, -1, -2 ** 31
    valid = torch.ones(T, dtype=torch.uint8)
    t, rc = bl.call(bl.handle("bf16", F, E, k, flags), u.cuda(), W.cuda(), idx.cuda(), None, T, F, E)
    assert rc == want
    assert torch.equal(t["counts"].cpu().long(), bl.reference(u, W, idx, valid, E, k)["counts"])


def test_captured_and_accumulated():
    T, F, E, k = 9000, 512, 16, 2
    u, W, idx, valid = bl.make("bf16", T, F, E, k, seed=6)
    h = bl.handle("bf16", F, E, k)
    mag = bl.reference(u, W, idx, valid, E, k)["dW_mag"].cuda()
    u, W, idx, valid = u.cuda(), W.cuda(), idx.cuda(), valid.cuda()
    want, rc = bl.call(h, u, W, idx, valid, T, F, E)
    assert rc == 0
    w = sb.make_weights(W, None, None, None, None)
    t = {n: torch.zeros_like(x) for n, x in want.items()}
    ws = torch.empty(sb.swimba_balance_loss_workspace_bytes(h, T), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sb.swimba_balance_loss(h, w, u, idx, valid, T, bl.COEF, t["loss"], t["counts"], t["mean"], t["dW"], t["du"], ws,
                               accumulate=True)
    for n in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[x], t[x]) for x in ("loss", "counts", "mean", "du"))
        # either side adds the same eight runs of partial sums n times: as many roundings of a running sum that stays
        # within n times the result and the magnitudes of one call's terms (and those twice over, for their own rounding)
        assert bool(((t["dW"] - n * want["dW"]).abs() <= 16 * n * 2.0 ** -24 * (n * want["dW"].abs() + 2 * mag)).all())


def test_the_same_expert_twice():
    """A token whose active set names an expert twice counts it twice, in either form of the counts."""
    for T, F, E, k in ((500, 256, 8, 2), (9000, 256, 8, 2), (300, 264, 40, 3)):
        u, W, idx, valid = bl.make("bf16", T, F, E, k, seed=T)
        idx[:, 0] = idx[:, -1]
        t, rc = bl.call(bl.handle("bf16", F, E, k), u.cuda(), W.cuda(), idx.cuda(), valid.cuda(), T, F, E)
        assert rc == 0
        bl.check(t, bl.reference(u, W, idx, valid, E, k), "bf16", T, F, E)
