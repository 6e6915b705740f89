"""The operators beside the mixer at the ends of their ranges, without a device: what is beyond is refused before anything is
planned with it, and the workspace queries give zero."""
import pytest

from paper_2603_06938_b200 import binding as sb
from test_operator_refusals import SHAPE, attention, gradient, handle, step

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
