"""The operators beside the mixer at the ends of their ranges, without a device: what is beyond is refused before anything is
planned with it, and the workspace queries give zero."""
import pytest

from paper_2603_06938_b200 import binding as sb
import test_operator_refusals as refusals
from test_operator_refusals import SHAPE, attention, gradient, step



def handle(**kw):
    """As there, on a device that no machine has: a call that is not refused for its sizes is refused for that."""
    block, h = refusals.handle(**kw)
    assert block[10] == 0 and block[11] == 148
    block[10] = 1 << 20
    return block, h


QUERIES = ("swimba_linear_attention_workspace_bytes", "swimba_linear_attention_backward_workspace_bytes")


@pytest.mark.parametrize("dtype", [sb.DTYPE_BF16, sb.DTYPE_FP32])
@pytest.mark.parametrize("B,L", [(1, 2 ** 31 - 1), (1, 2 ** 30 + 1), (2, 2 ** 30), (65536, 1), (2 ** 31 - 1, 1),
                                 (2 ** 31 - 1, 2 ** 31 - 1), (65535, 2 ** 15 + 1)])
def test_more_tokens_than_the_kernels_count(B, L, dtype):
    block, h = handle(dtype=dtype)
    for call in (attention, gradient):
        assert call(h, B=B, L=L) == SHAPE
        assert sb.lib().swimba_last_error(h)
    for f in QUERIES:
        assert getattr(sb.lib(), f)(h, B, L) == 0


def test_the_largest_sizes_have_a_plan():
    for dtype in (sb.DTYPE_BF16, sb.DTYPE_FP32):
        for H in (1, 4, 256):
            block, h = handle(H=H, G=1, dtype=dtype)
            for B, L in ((1, 2 ** 30), (1, 2 ** 30 - 127), (65535, 2 ** 15)):
                for f in QUERIES:
                    n = getattr(sb.lib(), f)(h, B, L)
                    assert n >= B * H * 64 * 128 * 4                # (a copy of the states at least)


@pytest.mark.parametrize("dtype", [sb.DTYPE_BF16, sb.DTYPE_FP32])
@pytest.mark.parametrize("ld,L", [(2 ** 31, 256), (2 ** 31, 4096), (2 ** 30, 512), (2 ** 29, 2 ** 20)])
def test_sequences_that_no_tensor_map_reaches(ld, L, dtype):
    block, h = handle(dtype=dtype)
    for call in (attention, gradient):
        for n in ("ldq", "ldk", "ldv"):
            assert call(h, B=1, L=L, **{n: ld}) == SHAPE
            assert b"2^40" in sb.lib().swimba_last_error(h)
            assert call(h, B=1, L=1, **{n: ld}) not in (SHAPE, sb.OK)          # (one token is refused for the device)
    assert step(h, B=2, ldq=ld) not in (SHAPE, sb.OK)
