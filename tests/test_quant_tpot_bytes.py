"""Cache bytes that the decode step's report names (paper_2606_00024_amd.tpot)."""
from __future__ import annotations

import pytest
import torch

from paper_2606_00024_amd import api, tpot


@pytest.mark.parametrize("kv,dtype", [("e4m3", torch.float8_e4m3fn), ("int8", torch.int8)])
@pytest.mark.parametrize("seq_len", [64, 640, 650])
def test_kv_bytes_are_those_of_the_caches(kv, dtype, seq_len):
    """Codes of the tokens and the scales of their runs, as new_quant_cache lays
    them out for pages of 64."""
    model = tpot.ModelShape("tiny", layers=3, hidden=512, q_heads=8, kv_heads=2, ffn=1024, vocab=1000)
    pages = -(-seq_len // 64)
    c = api.new_quant_cache(5 * pages, 2, 64, dtype=dtype, device="cpu")
    held = c.k.numel() * seq_len // (64 * pages) + c.k_scale.numel() * 4
    assert model.kv_bytes(5, seq_len, kv) == 3 * 2 * held
    assert model.kv_bytes(5, seq_len) == 3 * 2 * 2 * 5 * 2 * seq_len * 128
