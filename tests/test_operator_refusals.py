"""What the operators beside the mixer refuse, and their workspace queries, without a device: a refused call enqueues
nothing, so the pointers are never followed."""
import ctypes

import pytest

from paper_2603_06938_b200 import binding as sb
from paper_2603_06938_b200 import build as sbuild


def handle(F=64, H=4, P=64, N=128, G=2, E=4, k=2, dtype=sb.DTYPE_BF16):
    sbuild.build()
    block = (ctypes.c_int32 * 4096)(F, H, P, N, G, E, k, 128, dtype, 0, 0, 148)
    return block, ctypes.cast(block, ctypes.c_void_p)


A = 0x1000                      # an aligned address that no call gets to


def attention(h, log_decay=A, q=A, ldq=256, k=A, ldk=256, v=A, ldv=256, s_in=None, B=2, L=300, scale=1.0, o=A, s_out=None,
              ws=A, n=1 << 40):
    return sb.lib().swimba_linear_attention(h, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, L, scale, o, s_out, ws, n, None)


def gradient(h, log_decay=A, q=A, ldq=256, k=A, ldk=256, v=A, ldv=256, s_in=None, do=A, ds=None, B=2, L=300, scale=1.0,
             dq=A, dk=A, dv=A, ds_in=None, ws=A, n=1 << 40):
    return sb.lib().swimba_linear_attention_backward(h, log_decay, q, ldq, k, ldk, v, ldv, s_in, do, ds, B, L, scale, dq, dk,
                                                     dv, ds_in, ws, n, None)


def step(h, log_decay=A, q=A, ldq=256, k=A, ldk=256, v=A, ldv=256, s_in=A, B=2, scale=1.0, o=A, s_out=A):
    return sb.lib().swimba_linear_attention_step(h, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, scale, o, s_out, None)


def norm(h, x=A, ldx=256, w=A, b=A, rows=5, groups=4, width=64, eps=1e-5, y=A, mean=A, rstd=A):
    return sb.lib().swimba_layer_norm(h, x, ldx, w, b, rows, groups, width, eps, y, mean, rstd, None)


def norm_backward(h, dy=A, x=A, ldx=256, w=A, mean=A, rstd=A, rows=5, groups=4, width=64, dx=A, dw=A, db=A, ws=A, n=1 << 40):
    return sb.lib().swimba_layer_norm_backward(h, dy, x, ldx, w, mean, rstd, rows, groups, width, dx, dw, db, ws, n, None)


def balance(h, W=A, u=A, idx=A, valid=None, T=100, coef=0.01, loss=A, counts=A, mean=A, dW=A, add=0, du=A, ws=A, n=1 << 40):
    w = sb.swimba_weights()
    w.W_router = W
    return sb.lib().swimba_balance_loss(h, ctypes.byref(w), u, idx, valid, T, coef, loss, counts, mean, dW, add, du, ws, n,
                                        None)


NULL, SHAPE, ALIGN, SMALL = sb.ERR_NULL_ARG, sb.ERR_UNSUPPORTED_SHAPE, sb.ERR_MISALIGNED, sb.ERR_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("call", [attention, gradient, step, norm, norm_backward, balance])
def test_no_handle(call):
    assert call(None) == NULL


@pytest.mark.parametrize("call,arg,value,code", [
    *((c, n, None, NULL) for c in (attention, gradient, step) for n in ("log_decay", "q", "k", "v")),
    *((attention, n, None, NULL) for n in ("o", "ws")), *((step, n, None, NULL) for n in ("s_in", "s_out", "o")),
    *((gradient, n, None, NULL) for n in ("do", "dq", "dk", "dv", "ws")),
    *((c, n, 255, SHAPE) for c in (attention, gradient, step) for n in ("ldq", "ldk", "ldv")),
    *((c, n, 257, ALIGN) for c in (attention, gradient, step) for n in ("ldq", "ldk", "ldv")),
    *((c, n, A + 8, ALIGN) for c in (attention, gradient, step) for n in ("log_decay", "q", "k", "v", "s_in")),
    *((attention, n, A + 8, ALIGN) for n in ("o", "s_out", "ws")),
    *((gradient, n, A + 8, ALIGN) for n in ("do", "ds", "dq", "dk", "dv", "ds_in", "ws")),
    *((c, "B", v, SHAPE) for c in (attention, gradient, step) for v in (-1, 65536)),
    *((c, "L", v, SHAPE) for c in (attention, gradient) for v in (-1, 2 ** 31 - 1)),
    *((c, "n", 16, SMALL) for c in (attention, gradient)),
    *((norm, n, None, NULL) for n in ("x", "y")), *((norm_backward, n, None, NULL) for n in ("dy", "x", "mean", "rstd", "dx", "ws")),
    *((norm, n, A + 4, ALIGN) for n in ("x", "w", "b", "y", "mean", "rstd")),
    *((norm_backward, n, A + 4, ALIGN) for n in ("dy", "x", "w", "mean", "rstd", "dx", "dw", "db", "ws")),
    *((c, n, v, SHAPE) for c in (norm, norm_backward) for n, v in (("rows", -1), ("groups", 0), ("width", 0), ("width", 60),
                                                                   ("width", 16392), ("groups", 70000), ("ldx", 255))),
    *((c, "ldx", 260, ALIGN) for c in (norm, norm_backward)), (norm_backward, "n", 16, SMALL),
    *((balance, n, None, NULL) for n in ("W", "u", "idx", "loss", "ws")),
    *((balance, n, A + 4, ALIGN) for n in ("W", "u", "idx", "loss", "counts", "mean", "dW", "du", "ws")),
    (balance, "T", -1, SHAPE), (balance, "T", 1 << 30, SHAPE), (balance, "n", 16, SMALL)])
def test_refused(call, arg, value, code):
    block, h = handle()
    assert call(h, **{arg: value}) == code
    assert sb.lib().swimba_last_error(h)


def test_head_sizes_the_kernels_lack():
    block, h = handle(P=20, N=32)
    for call in (attention, gradient, step):
        assert call(h, ldv=128) == SHAPE


def test_nothing_to_do():
    block, h = handle()
    for call in (attention, gradient):
        assert call(h, B=0, q=None) == 0 and call(h, L=0, ws=None) == 0
    assert step(h, B=0, s_in=None) == 0 and norm(h, rows=0, x=None) == 0 and balance(h, T=0, u=None) == 0


def test_workspaces_grow():
    lib = sb.lib()
    for args in (dict(), dict(H=1, G=1), dict(H=16, G=16, N=64), dict(H=3, G=3, N=32, P=48), dict(dtype=sb.DTYPE_FP32)):
        block, h = handle(**args)
        for f in (lib.swimba_linear_attention_workspace_bytes, lib.swimba_linear_attention_backward_workspace_bytes):
            for B in (1, 2, 3, 9):
                sizes = [f(h, B, L) for L in (*range(1, 2000, 61), *range(2000, 90000, 3001))]
                assert sizes == sorted(sizes) and sizes[0] > 0
            for L in (1, 64, 200, 1500, 30000):
                sizes = [f(h, B, L) for B in range(1, 70)]
                assert sizes == sorted(sizes)
            assert f(h, 0, 5) == 0 and f(h, 5, 0) == 0 and f(None, 1, 1) == 0
        sizes = [lib.swimba_balance_loss_workspace_bytes(h, T) for T in range(1, 40000, 97)]
        assert sizes == sorted(sizes)
        assert lib.swimba_balance_loss_workspace_bytes(h, 1 << 31) == 0
    assert lib.swimba_layer_norm_workspace_bytes(h, 10, 1, 60) == 0
