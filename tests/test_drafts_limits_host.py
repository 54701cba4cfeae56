"""Sizes of the calls on drafted tokens that are refused before a launch (no GPU)."""
from __future__ import annotations

import pytest

from paper_2606_00024_amd import _lib
from test_drafts_host import NO, PTR, _append, _rope_rows, _rows, _shape


@pytest.mark.parametrize("heads", [1 << 28, 1 << 30, 2 ** 31 - 1])
def test_heads_past_32_bits_are_refused(heads):
    """q, k and v together, and a step past the last, would leave 32 bits."""
    many = _rows(heads, stride_row=0, stride_head=0)
    assert _rope_rows(x_rows=many, out_rows=many) == NO
    assert _append(_shape(num_kv_heads=heads, num_q_heads=heads), k_rows=many, v_rows=many) == NO
    assert _append(_shape(num_q_heads=heads), q=PTR, q_out=PTR, q_rows=many, q_out_rows=many) == NO
