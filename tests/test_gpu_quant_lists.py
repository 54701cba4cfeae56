"""Block lists over an 8-bit cache (needs a gfx950 GPU): the layouts that
decode_attention takes."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import quantref as R
from helpers import small_workload
from paper_2606_00024_amd import _lib, api

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


@pytest.mark.parametrize("no_detector", [False, True])
def test_shared_lists_in_either_layout(no_detector):
    """One list a sequence as [batch][1][n] or [batch][n], with lengths of either
    form: the same bits, and those of the same lists per head."""
    wl = small_workload(81, batch=3, kv_heads=2, group=4, seq_len=(900, 0, 640), needles=2)
    cache, plain = R.quantised(wl, "e4m3", 32)
    cache = R.to_device(cache, DEV)
    rng = np.random.default_rng(81)
    lists, counts = np.full((3, 15), -1, dtype=np.int32), np.array([9, 0, 10], dtype=np.int32)
    for b, n in ((0, 15), (2, 10)):
        lists[b, : counts[b]] = rng.permutation(n)[: counts[b]]
    bl, bll = torch.from_numpy(lists).to(DEV), torch.from_numpy(counts).to(DEV)
    args = [t.to(DEV) for t in (plain.page_table, plain.seq_lens)]

    def call(lists, counts, per_head):
        return api.decode_attention_quant(plain.q.to(DEV), cache, *args, block_size=64, tau=0.02, phi=0.02,
                                          patience=2, no_detector=no_detector, block_list=lists,
                                          block_list_len=counts, list_per_head=per_head)

    want = call(bl[:, None].expand(3, 2, 15).contiguous(), bll[:, None].expand(3, 2).contiguous(), True)
    assert want[2].max() > 0
    for got in (call(bl, bll, False), call(bl[:, None], bll, False), call(bl[:, None], bll[:, None], False),
                call(bl, bll[:, None], False)):
        for a, b in zip(want, got):
            assert torch.equal(a, b)
    with pytest.raises(ValueError, match="block_list"):
        call(bl[:2], bll, False)
    with pytest.raises(ValueError, match="block_list"):
        call(bl[:, None], bll, True)
    with pytest.raises(ValueError, match="block_list_len"):
        call(bl, bll[:2], False)
    with pytest.raises(ValueError, match="block_list"):
        call(bl.t().contiguous().t(), bll, False)
