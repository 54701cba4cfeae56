"""Calls on drafted tokens where a sequence's slots pass 2^31, in tables that have
room for them (needs a gfx950 GPU)."""
from __future__ import annotations

import pytest
import torch

from paper_2606_00024_amd import _lib, api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PAGE = 1 << 16
FAR = 2 ** 31


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


class FarCache:
    """Two sequences whose table goes a few pages past slot 2^31; the pages around it
    exist, all others are marked as missing."""

    def __init__(self, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.k, self.v = (torch.randn(4, 2, PAGE, 128, generator=gen, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        self.table = torch.full((2, FAR // PAGE + 3), -1, dtype=torch.int32, device=DEV)
        for b in range(2):
            self.table[b, FAR // PAGE - 1], self.table[b, FAR // PAGE] = 2 * b + 1, 2 * b

    def rows(self, pool, b, slots):
        """The rows [slots][heads][128] of a pool."""
        return torch.stack([pool[int(self.table[b, t // PAGE]), :, t % PAGE] for t in slots])


def test_accepted_nodes_move_across_2_to_the_31():
    c = FarCache(1)
    was = {name: getattr(c, name).clone() for name in "kv"}
    paths = [[0, 2, 4, 5], [1, 3, 4]]
    held = [FAR - 3, FAR - 1]
    accepted = torch.tensor([p + [-1] * (4 - len(p)) for p in paths], dtype=torch.int32, device=DEV)
    counts = torch.tensor([len(p) for p in paths], dtype=torch.int32, device=DEV)
    api.keep_accepted(c.k, c.v, c.table, torch.tensor(held, dtype=torch.int32, device=DEV), accepted, counts)
    for name in "kv":
        want = was[name].clone()
        for b, path in enumerate(paths):
            for j, node in enumerate(path):
                to = held[b] + j
                want[int(c.table[b, to // PAGE]), :, to % PAGE] = c.rows(was[name], b, [held[b] + node])[0]
        assert torch.equal(getattr(c, name), want)


def test_appended_keys_turn_by_positions_past_2_to_the_31():
    """Without row_positions a row's position is its slot: 2^31 and further are no
    negative numbers.  A frequency of 2^-34 turns slot 2^31 by 1/8 rad (and -2^31 by
    -1/8).  Bound: 2^-21 of |x| + |y| in fp32, and a rounding to bf16 of 2^-8."""
    c = FarCache(2)
    freqs = torch.full((64,), 2.0 ** -34, dtype=torch.float64, device=DEV)
    x = torch.randn(10, 2, 128, generator=torch.Generator().manual_seed(3))
    held = [FAR - 2, FAR - 3]
    rows = x.to(DEV)
    q = api.rope_append(c.k, c.v, rows, rows, c.table, torch.tensor(held, dtype=torch.int32, device=DEV),
                        rope=api.Rope(freqs), q=rows)
    for b in range(2):
        slots = [held[b] + i for i in range(5)]
        at, y = torch.tensor(slots, dtype=torch.float64)[:, None, None] * 2.0 ** -34, x[5 * b: 5 * b + 5].double()
        lo, hi = y[..., :64], y[..., 64:]
        want = torch.cat([lo * at.cos() - hi * at.sin(), hi * at.cos() + lo * at.sin()], -1)
        size = (lo.abs() + hi.abs()).repeat(1, 1, 2)
        for got in (c.rows(c.k, b, slots), q[5 * b: 5 * b + 5]):
            assert bool(((got.cpu().double() - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * size).all())
        assert torch.equal(c.rows(c.v, b, slots), rows[5 * b: 5 * b + 5].bfloat16())


def test_layouts_whose_positions_32_bits_do_not_hold_are_passed_over():
    parents = torch.tensor([-1, 0, 1, 2] * 3, dtype=torch.int32, device=DEV)
    context = torch.tensor([FAR - 4, FAR - 3, FAR - 1], dtype=torch.int32, device=DEV)
    mask = torch.full((12, 1), 9, dtype=torch.int64, device=DEV)
    positions = torch.full((12,), 9, dtype=torch.int32, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    args = (3, 12, parents.data_ptr(), 0, context.data_ptr(), 1, mask.data_ptr())
    assert _lib.tree_layout(*args, positions.data_ptr(), stream) == _lib.OK
    assert positions.tolist() == [FAR - 4, FAR - 3, FAR - 2, FAR - 1] + [9] * 8
    assert mask[:, 0].tolist() == [1, 3, 7, 15] + [9] * 8
    # bits alone have no such bound
    assert _lib.tree_layout(*args, 0, stream) == _lib.OK
    assert mask[:, 0].tolist() == [1, 3, 7, 15] * 3
