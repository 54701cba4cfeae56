"""Attention of drafted tokens: values that are not finite behind scores of -inf,
offsets that claim rows many times over, and what a bf16 output rounds (needs a
gfx950 GPU)."""
from __future__ import annotations

import math

import pytest
import torch

import draftref as R
from paper_2606_00024_amd import _lib, api
from test_gpu_tree import DEV, DTYPES, LONG, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


def _put(pool, table, tokens, dim, x):
    """Dim `dim` (or all) of these tokens of sequence 0."""
    for t in tokens:
        pool[table[0, t // 16].long(), :, t % 16, dim] = x


ALL = slice(None)
# held, new, heads, columns of the table behind the sequence's: row tiles of 32, 64 and 128
# rows, in one workgroup and split over many
SHAPES = [(50, 5, (4, 2), LONG), (9000, 3, (2, 1), LONG), (300, 9, (4, 2), 0), (9000, 30, (2, 1), 0),
          (40, 40, (8, 1), 0), (2000, 40, (8, 1), 0)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("held, new, heads, extra", SHAPES, ids=str)
def test_values_behind_scores_of_minus_infinity(held, new, heads, extra, dtype):
    """Tokens whose keys make every score -inf are unseen, whatever their values: the
    same bits as with values of 0 there, and what the definition has without them.
    The first stretch of the context is of such tokens alone."""
    p = Problem([held], [new], heads, seed=31, extra_width=extra)
    p.q[..., 9] = p.q[..., 9].abs() + 0.5
    table = p.cache.table
    gone = list(range(held // 4)) + [held // 2, held - 1]
    _put(p.cache.k, table, gone, 9, 0.0)
    _put(p.cache.v, table, gone, ALL, 0.0)
    work = R.attend(p.q, p.cache.k, p.cache.v, table, p.context, p.offsets, p.mask, p.scale)[3]
    _put(p.cache.k, table, gone, 9, -math.inf)
    plain = p.run(dtype)
    cache = p.cache.to(DEV)
    for i, t in enumerate(gone):
        _put(cache.v, cache.table, [t], ALL, (math.inf, math.nan, -math.inf)[i % 3])
    out, lse = p.run(dtype, cache=cache)
    assert torch.equal(out, plain[0]) and torch.equal(lse, plain[1])
    ref, ref_lse, size, _, count = R.attend(p.q, p.cache.k, p.cache.v, table, p.context, p.offsets, p.mask, p.scale)
    far, far_lse = R.attend_bounds(ref, ref_lse, size, work, count, dtype is torch.bfloat16)
    live = slice(p.lead, -p.lead)
    assert bool(((out.double().cpu() - ref).abs() <= far)[live].all())
    assert bool(((lse.double().cpu() - ref_lse).abs() <= far_lse)[live].all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("held, new, heads, extra", SHAPES, ids=str)
def test_rows_whose_scores_are_all_minus_infinity(held, new, heads, extra, dtype):
    p = Problem([held], [new], heads, seed=32, extra_width=extra)
    p.q[..., 9] = p.q[..., 9].abs() + 0.5
    _put(p.cache.k, p.cache.table, range(held + new), 9, -math.inf)
    _put(p.cache.v, p.cache.table, range(0, held + new, 7), ALL, math.nan)
    out, lse = (x[p.lead: -p.lead] for x in p.run(dtype))
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("held, new, heads, extra", SHAPES, ids=str)
def test_a_value_that_some_rows_see(held, new, heads, extra, dtype):
    """A score that overflows to -inf in the even nodes, and is finite in the odd ones,
    if of weight 0: those get the infinite value."""
    p = Problem([held], [new], heads, seed=33, extra_width=extra)
    even = torch.arange(p.lead, p.lead + new, 2)
    odd = torch.arange(p.lead + 1, p.lead + new, 2)
    p.q[..., 9] = 1e-6
    p.q[even, :, 9] = 100.0
    _put(p.cache.k, p.cache.table, [held // 2], 9, -3e38)
    _put(p.cache.v, p.cache.table, [held // 2], ALL, 0.0)
    plain = p.run(dtype)
    cache = p.cache.to(DEV)
    _put(cache.v, cache.table, [held // 2], 77, -math.inf)
    out, lse = p.run(dtype, cache=cache)
    assert torch.equal(out[even], plain[0][even]) and torch.equal(lse, plain[1])
    assert bool((out[odd][..., 77] == -math.inf).all())
    others = [d for d in range(128) if d != 77]
    assert torch.equal(out[odd][..., others], plain[0][odd][..., others])


@pytest.mark.parametrize("heads, batch, rows, extra", [((128, 1), 40, 8, 300), ((256, 2), 100, 100, LONG), ((8, 1), 300, 600, 40)])
def test_offsets_that_claim_rows_many_times(heads, batch, rows, extra):
    """0, rows, 0, rows, ...: half of the sequences claim every row, more units of work
    than any offsets that do not decrease can make.  Nothing is written, and the next
    call over the same workspace is as ever."""
    p = Problem([20] * batch, [rows // batch or 1] * batch, heads, seed=34, extra_width=extra, tree=False, offsets=None)
    p.q = p.q[:rows]
    p.offsets = torch.tensor([rows * (b % 2) for b in range(batch + 1)], dtype=torch.int32)
    workspace = torch.empty(128 << 20, dtype=torch.uint8, device=DEV)
    out, lse = p.run(torch.float32, workspace=workspace)
    assert bool((out == 77).all()) and bool((lse == 77).all())
    fine = Problem([700, 30], [9, 3], (8, 2), seed=35)
    want, got = fine.run(torch.float32), fine.run(torch.float32, workspace=workspace)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("held, new, heads, extra", [([300], [3], (4, 2), LONG), ([900, 40], [2, 4], (8, 2), LONG),
                                                     ([300], [9], (4, 2), 0), ([700, 33], [5, 5], (8, 1), 0)], ids=str)
def test_bf16_outputs_of_few_rows_are_rounded_once(held, new, heads, extra, tree):
    """Up to 64 rows to a KV head (the packed rows, unused ones too, over the batch, times
    the group: 18, 24, 30 and 64 here): probabilities carry 16 bits (two roundings
    to bf16 of what the one before leaves: 2^-16), so that outputs near 0, where values
    cancel, are as close as the output's own rounding (2^-8) lets them be."""
    p = Problem(held, new, heads, seed=36, extra_width=extra, tree=tree)
    out, _ = p.run(torch.bfloat16)
    ref, ref_lse, size, work, count = R.attend(p.q, p.cache.k, p.cache.v, p.cache.table, p.context, p.offsets, p.mask, p.scale)
    far = R.attend_bounds(ref, ref_lse, size, work, count, False)[0] + 2.0 ** -16 * size
    far = far + 2.0 ** -8 * (ref.abs() + far)
    live = slice(p.lead, -p.lead)
    assert bool(((out.double().cpu() - ref).abs() <= far)[live].all())
