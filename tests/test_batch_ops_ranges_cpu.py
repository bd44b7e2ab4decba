"""Refusals of the batch operators at the ends of their ranges; no GPU needed.  A refused call touches nothing, so the
pointers here are never followed."""
import pytest

from paper_2606_03113_amd import lede
from tests.test_batch_ops_cpu import ATTN, ATTN_GOOD, _change, lib  # noqa: F401


@pytest.mark.parametrize("scale", [1.1e38, -1.1e38, 3.4e38, -3.4e38], ids=str)
def test_attention_refuses_scales_beyond_its_range(lib, scale):  # noqa: F811
    """In the exponent's base the scale is 2 log2(e) times as large: from 1.2e38 on it would be infinite there."""
    assert lib.lede_op_cache_attention(*_change(ATTN_GOOD, ATTN, scale=scale)) == lede.LEDE_E_ARG
    assert lib.lede_op_cache_attention(*_change(ATTN_GOOD, ATTN, scale=scale / 4, n_rows=0)) == 0
