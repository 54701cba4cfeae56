"""Chunk lengths of walks with the test over an 8-bit cache (no GPU): the plans
of 16 heads and of few long groups are chosen where planref says, seen from the
workspace bytes that their chunks take."""
from __future__ import annotations

import os

import pytest

import planref
from paper_2606_00024_amd import _lib
from test_gpu_quant_plans import PLANS
from test_quant_host import _decode, _opts, _shape, _spec

# g, groups, blocks of the longest traversal, tokens of a block, blocks in a chunk
CASES = [
    (16, 4, 127, 64, 3), (16, 4, 128, 64, 9), (16, 256, 200, 64, 9), (16, 4, 900, 64, 9), (16, 64, 300, 128, 6),
    (16, 8, 127, 128, 3), (16, 16, 64, 256, 3), (16, 16, 140, 256, 6), (16, 4, 200, 512, 6), (16, 4, 200, 1024, 3),
    (8, 8, 767, 64, 9), (8, 8, 768, 64, 15), (8, 9, 768, 64, 9), (8, 1, 768, 64, 12), (8, 8, 800, 128, 15),
    (4, 8, 768, 64, 15), (4, 2, 1000, 64, 15), (4, 9, 1000, 64, 9), (2, 1, 2000, 64, 15), (1, 8, 768, 64, 15),
    (1, 1, 768, 64, 12), (4, 8, 800, 512, 6), (4, 64, 512, 64, 9), (1, 64, 512, 64, 9),
]


@pytest.mark.parametrize("g,groups,t,block,length", CASES + [p[:5] for p in PLANS])
def test_chunk_lengths(g, groups, t, block, length):
    assert planref.chunks(g, groups, t, block)[0] == length
    if os.path.exists("/dev/kfd"):
        pytest.skip("a GPU is visible: calls that pass the checks launch with placeholder pointers")
    shape = _shape(batch=groups, num_kv_heads=1, num_q_heads=g, block_size=block, num_pages=1 << 20,
                   max_pages_per_seq=t * block // 64)
    least = planref.least_bytes(g, groups, t, block)
    assert least <= _lib.workspace_bytes(shape, _opts())
    assert _decode(shape, _opts(), _spec(), workspace_bytes=least) == _lib.ERR_HIP
    assert _decode(shape, _opts(), _spec(), workspace_bytes=least - 1) == _lib.ERR_WORKSPACE_TOO_SMALL
