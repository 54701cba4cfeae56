"""Attention of drafted tokens where every workgroup goes through many tiles: pages in
random order, page ids asked for again and again, against the definition in 64 bits
(needs a gfx950 GPU).

Bounds.  A matrix instruction adds its 16 products to the sum in two roundings of
2^-24, and an fp32 output has three for 16 tokens; a row's sum has one rounding for 32
tokens, and 16 within them.  Scores as in draftref.attend_bounds."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2606_00024_amd import _lib, api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PAGE = 64


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


def longest_segments(batch, rows, kv_heads, group, width, seen):
    """(blocks of 32 rows of a row tile, tiles of the longest segment of every workgroup):
    the plan and the cut of the line, for sequences of one row tile each."""
    cap, per = width * PAGE, -(-rows // batch) * group
    units = batch * kv_heads
    few = per <= 32 and group <= 32 and units <= 512 and units * -(-cap // 128) >= 512
    rb = 1 if few else 2 if per <= 64 and group <= 64 else 4
    tile, lead, least = {1: (128, 2, 1), 2: (64, 4, 2), 4: (32, 4, 2)}[rb]
    most = 256 if rb == 1 else 512
    at_most = kv_heads * (rows // (32 * rb // group) + batch)
    grid = min(at_most * -(-cap // tile) if at_most < most else at_most, most)
    starts, line = [], 0
    for n in seen:
        for _ in range(kv_heads):
            starts.append((line, -(-n // tile)))
            line += lead + starts[-1][1]
    workers = min(grid, max(line // least, 1))
    longest = []
    for me in range(workers):
        begin, end = me * line // workers, (me + 1) * line // workers
        longest.append(max((min(end, s + lead + n) - max(begin, s + lead) for s, n in starts if s < end and begin < s + lead + n), default=0))
    return rb, longest


class Long:
    """Sequences over a small pool of pages, each in an order of its own.  Two tokens of
    every page have a score that makes them weigh as much as all others together."""

    def __init__(self, batch, nodes, group, lo, hi, *, tree, seed, heads=8):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)  # noqa: E731
        number = lambda lo, hi, *shape: torch.randint(lo, hi + 1, shape, generator=gen, device=DEV)  # noqa: E731
        self.nodes, self.group, self.heads = nodes, group, heads
        self.context = number(lo, hi, batch).int()
        width = -(-(hi + nodes) // PAGE)
        self.table = number(0, 47, batch, width).int()
        u = normal(heads, 128)
        u = u / u.norm(dim=-1, keepdim=True) * math.sqrt(128)
        self.k, self.v = normal(48, heads, PAGE, 128), normal(48, heads, PAGE, 128).bfloat16()
        for slot in (number(0, 31, 48), number(32, 63, 48)):
            self.k[torch.arange(48, device=DEV), :, slot] += 0.5 * u
        self.k = self.k.bfloat16()
        q = normal(batch, nodes, heads, group, 128) * 0.5 + u[:, None]
        self.q = q.view(batch * nodes, heads * group, 128).bfloat16()
        self.mask = None
        if tree:
            self.mask = number(0, 2 ** nodes - 1, batch * nodes, 1) | 1

    def run(self, dtype, **kw):
        args = {"v": self.v, **kw}
        return api.tree_attention(self.q, self.k, args["v"], self.table, self.context, mask=self.mask, out_dtype=dtype)

    def check(self, out, lse, dtype, dims=slice(None)):
        """Sixteen sequences' heads in fp64."""
        batch, n, g = len(self.context), self.nodes, self.group
        out, lse = out.view(batch, n, self.heads, g, 128), lse.view(batch, n, self.heads, g)
        worst = 0.0
        for i in range(16):
            b, h = i * (batch - 1) // 15, i * 5 % self.heads
            c = int(self.context[b])
            pages = self.table[b].long()
            keys, values = (x[pages, h].reshape(-1, 128)[: c + n].double() for x in (self.k, self.v))
            q = self.q.view(batch, n, self.heads, g, 128)[b, :, h].double().reshape(n * g, 128)
            node = torch.arange(c + n, device=DEV) - c
            own = torch.arange(n, device=DEV)[:, None]
            if self.mask is None:
                sees = node <= own
            else:
                sees = (node < 0) | (self.mask.view(batch, n)[b][:, None] >> node.clamp_min(0) & 1).bool()
            s = (q @ keys.T / math.sqrt(128)).view(n, g, -1).masked_fill(~sees[:, None], -math.inf)
            ref_lse = torch.logsumexp(s, -1)
            w = torch.exp(s - ref_lse[..., None]).view(n * g, -1)
            ref, size = (w @ values).view(n, g, 128), (w @ values.abs()).view(n, g, 128)
            work = float((q.abs() @ keys.abs().T).max()) / math.sqrt(128) / math.log(2)
            score = math.log(2) * 133 * work * 2.0 ** -24 + 2.0 ** -22
            bf16 = dtype is torch.bfloat16
            sums = ((0.375 + 1 / 32) * (c + n) + 48) * 2.0 ** -24
            far = size * (2 * (score + sums) + (2.0 ** -8 if bf16 else 2.0 ** -22))
            if bf16:
                far = far + 2.0 ** -8 * (ref.abs() + far)
            far_lse = score + sums + 2.0 ** -21 * (ref_lse.abs() + 1)
            for got, want, bound in ((out[b, :, h].double()[..., dims], ref[..., dims], far[..., dims]), (lse[b, :, h].double(), ref_lse, far_lse)):
                worst = max(worst, float(((got - want).abs() / bound).nan_to_num(1e9).max()))
        assert worst <= 1.0, worst


# row tiles of 32, 64 and 128 rows: sequences, nodes, group, contexts, tiles for which a
# wavefront's 64 lanes hold page ids
CASES = [(1, 32, 4, 8, 11500, 13500, 32), (2, 64, 8, 8, 11500, 13500, 64), (4, 64, 16, 8, 6000, 7500, 64)]


def _assert_long(p, rb, ahead):
    got, longest = longest_segments(len(p.context), len(p.q), p.heads, p.group, p.table.shape[1], [int(c) + p.nodes for c in p.context])
    assert got == rb and sorted(longest)[len(longest) // 2] > 2 * ahead


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("rb, batch, nodes, group, lo, hi, ahead", CASES, ids=["32", "64", "128"])
def test_many_tiles_a_workgroup(rb, batch, nodes, group, lo, hi, ahead, tree, dtype):
    p = Long(batch, nodes, group, lo, hi, tree=tree, seed=rb)
    _assert_long(p, rb, ahead)
    p.check(*p.run(dtype), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rb, batch, nodes, group, lo, hi, ahead", CASES, ids=["32", "64", "128"])
def test_many_tiles_with_values_that_are_not_finite(rb, batch, nodes, group, lo, hi, ahead, dtype):
    """One page holds an infinite value: parts of the line are gone through twice, from
    their first page ids on."""
    p = Long(batch, nodes, group, lo, hi, tree=True, seed=10 + rb)
    _assert_long(p, rb, ahead)
    p.table[p.table == 7] = 8
    p.table[:, 60], p.table[::2, 75] = 7, 7
    v = p.v.clone()
    v[7, :, 40, 99] = -math.inf
    out, lse = p.run(dtype, v=v)
    assert bool((out[..., 99] == -math.inf).all())
    p.check(out, lse, dtype, [d for d in range(128) if d != 99])


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("batch, nodes, held", [(256, 1, 32), (512, 8, 64), (512, 16, 128)], ids=["32", "64", "128"])
def test_sums_of_many_small_weights_behind_large_ones(batch, nodes, held, sign):
    """128 tokens of weight 1, then 16K of 0.3 steps of the sum that a wavefront holds of
    the first ones (32, 64 or 128 of them): one by one they would round away, out and
    lse.  Eight products are added at once, which may be off by half a step of their 2.4,
    and a row's sum takes 16 at once in half as large a sum, half a step of 9.6; a
    probability's lower parts (2^-8 of it) may be lost.  With values of -1 the sum falls
    below a power of two, where steps are half as large."""
    context, page, group = 16384, 128, 8
    weight = 0.3 * held * 2.0 ** -23
    scale = -math.log(weight) / 128
    pages = context // page + 1
    k = torch.zeros(pages, 1, page, 128, dtype=torch.bfloat16, device=DEV)
    k[1:, :, :, 0] = -8.0
    v = torch.ones_like(k)
    v[1:] = sign
    q = torch.zeros(batch * nodes, group, 128, dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = 16.0
    table = torch.arange(pages, dtype=torch.int32, device=DEV).expand(batch, pages).contiguous()
    lens = torch.full((batch,), context, dtype=torch.int32, device=DEV)
    out, lse = api.tree_attention(q, k, v, table, lens, softmax_scale=scale)
    small = (context - 128 + 1 + torch.arange(nodes, dtype=torch.float64)) * weight / 128
    ref = ((1 + sign * small) / (1 + small))[:, None, None]
    in_out, in_sum = 0.5 / 2.4 + 2.0 ** -8, 0.5 / 9.6
    few = 64 * 2.0 ** -24 + 2.0 ** -22 + 128 * scale * 2.0 ** -22 * float(small[-1])
    tail = float(small[-1])
    err = (out.cpu().double().view(batch, nodes, group, 128) - ref).abs().max().item()
    assert err <= (in_out + in_sum) * tail + few, (err, tail)
    err = (lse.cpu().double().view(batch, nodes, group) - torch.log(128 * (1 + small))[:, None]).abs().max().item()
    assert err <= in_sum * tail + few + 2 * 5 * 2.0 ** -23, (err, tail)
