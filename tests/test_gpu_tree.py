"""Attention of drafted tokens against its definition in 64 bits (needs a gfx950
GPU).  The bounds are draftref.attend_bounds's."""
from __future__ import annotations

import math

import pytest
import torch

import draftref as R
from paper_2606_00024_amd import _lib, api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


def _gpu_tensor(t):
    return None if t is None else t.to(DEV)


class Problem:
    def __init__(self, held, new, heads, *, page=16, tree=True, seed=0, offsets="ragged", pad=0, words=None, sharp=1.0,
                 extra_width=0):
        gen = torch.Generator().manual_seed(seed)
        self.gen = gen
        Hq, H = heads
        self.lead = 3 if offsets == "ragged" else 0
        rows = sum(new) + 2 * self.lead
        self.cache = R.Cache(gen, [a + b for a, b in zip(held, new)], H, page, pad=pad, extra_width=extra_width)
        self.q = (torch.randn(rows, Hq, 128, generator=gen) * sharp).bfloat16()
        self.context = torch.tensor(held, dtype=torch.int32)
        self.offsets = None
        if offsets == "ragged":
            self.offsets = torch.tensor([self.lead + sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32)
        self.parents = [R.random_parents(gen, n) for n in new]
        self.mask = None
        if tree:
            words = words or max(1, -(-max(new) // 64))
            lines = [R.bits(R.ancestors(p, i), words) for p in self.parents for i in range(len(p))]
            pad_lines = [[-1] * words for _ in range(self.lead)]
            self.mask = torch.tensor(pad_lines + lines + pad_lines, dtype=torch.int64)
        self.scale = 1 / math.sqrt(128)

    def run(self, dtype, cache=None, **kw):
        cache = cache or self.cache.to(DEV)
        rows, Hq, _ = self.q.shape
        out = torch.full((rows, Hq, 128), 77.0, dtype=dtype, device=DEV)
        lse = torch.full((rows, Hq), 77.0, device=DEV)
        return api.tree_attention(_gpu_tensor(self.q), cache.k, cache.v, cache.table, _gpu_tensor(self.context),
                                  mask=_gpu_tensor(self.mask), token_offsets=_gpu_tensor(self.offsets),
                                  softmax_scale=self.scale, out_dtype=dtype, out=out, lse=lse, **kw)

    def check(self, dtype=torch.float32, **kw):
        out, lse = (x.double().cpu() for x in self.run(dtype, **kw))
        ref, ref_lse, size, work, count = R.attend(self.q, self.cache.k, self.cache.v, self.cache.table, self.context,
                                                   self.offsets, self.mask, self.scale)
        idle = ref_lse[:, 0].isnan() & (count[:, 0] == 0)
        assert bool((out[idle] == 77).all()) and bool((lse[idle] == 77).all())
        live = ~idle
        empty = live & (count[:, 0] == 0)
        assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
        live &= ~empty
        far, far_lse = R.attend_bounds(ref, ref_lse, size, work, count, dtype is torch.bfloat16)
        for got, want, bound in ((out[live], ref[live], far[live]), (lse[live], ref_lse[live], far_lse[live])):
            bad = ~((got - want).abs() <= bound)
            assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, by up to {float(((got - want).abs() / bound).max()):.2f} of the bound"


DTYPES = [torch.float32, torch.bfloat16]
# Columns of the page table behind the sequences' own: with room for long contexts, and
# up to 32 rows a sequence, the row tiles are of 32 rows (of 64 without).
LONG = 4096


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("heads", [(1, 1), (4, 1), (8, 2), (5, 1), (32, 1), (9, 3)])
def test_row_tiles_of_32_rows(heads, tree, dtype):
    for i, (held, new) in enumerate((([0], [1]), ([1], [5]), ([127], [2]), ([128], [1]), ([129], [3]), ([700, 0, 33], [4, 1, 0]),
                                     ([5000], [3]), ([20, 300] * 6, [1, 2] * 6), ([64, 20], [11, 1]))):
        Problem(held, new, heads, tree=tree, seed=i, extra_width=LONG).check(dtype)


def test_hidden_values_in_row_tiles_of_32_rows():
    for new, heads in ((6, (4, 2)), (2, (16, 1))):
        for k_bad, v_bad in ((math.nan, math.nan), (0.0, math.inf)):
            p = Problem([150], [new], heads, seed=26, extra_width=LONG)
            others = torch.tensor([i for i in range(new) if i != new - 1]) + p.lead
            p.mask[others] &= ~(1 << (new - 1))
            clean = p.run(torch.float32)
            cache = p.cache.to(DEV)
            t = 150 + new - 1
            cache.k[cache.table[0, t // 16].long(), :, t % 16] = k_bad
            cache.v[cache.table[0, t // 16].long(), :, t % 16] = v_bad
            out, lse = p.run(torch.float32, cache=cache)
            assert torch.equal(out[others], clean[0][others]) and torch.equal(lse[others], clean[1][others])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads", [(1, 1), (8, 2), (6, 2), (5, 1), (16, 2), (16, 1), (40, 1)])
def test_heads(heads, dtype):
    for new in ([1], [4], [9]):
        Problem([130], new, heads, seed=heads[0]).check(dtype)


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("held", [[0], [1], [15], [16], [63], [64], [65], [127], [128], [129], [1000]])
def test_contexts(held, tree):
    for i, new in enumerate(([1], [5], [17], [40])):
        Problem(held, new, (4, 2), tree=tree, seed=i).check()


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("heads", [(4, 1), (8, 1), (3, 1), (32, 1)])
def test_many_nodes(heads, tree):
    """Several row tiles of a head, masks of several words."""
    Problem([70], [150], heads, tree=tree, seed=1, page=32).check(torch.bfloat16)
    Problem([0], [130], heads, tree=tree, seed=2).check()
    Problem([333], [65], heads, tree=tree, seed=3).check(torch.bfloat16)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tree", [True, False])
def test_ragged_batches(tree, dtype):
    Problem([0, 700, 33, 5, 2000, 64], [7, 1, 0, 33, 12, 64], (8, 2), tree=tree, seed=4).check(dtype)
    Problem([3] * 9, [2] * 9, (4, 4), tree=tree, seed=5, offsets=None).check(dtype)
    Problem([100, 0, 50] * 100, [1, 2, 3] * 100, (2, 1), tree=tree, seed=6).check(dtype)


@pytest.mark.parametrize("page", [16, 64, 256])
def test_pages_and_strides(page):
    Problem([500, 77], [20, 3], (8, 2), page=page, pad=1, seed=7).check()
    p = Problem([500, 77], [20, 3], (8, 2), page=page, seed=8)
    out, lse = p.run(torch.float32)
    wide = torch.zeros((p.q.shape[0], 12, 136), dtype=torch.bfloat16, device=DEV)
    wide[:, 2:10, :128] = p.q.to(DEV)
    c = p.cache.to(DEV)
    again = api.tree_attention(wide[:, 2:10, :128], c.k, c.v, c.table, p.context.to(DEV), mask=p.mask.to(DEV),
                               token_offsets=p.offsets.to(DEV), softmax_scale=p.scale)
    live = slice(p.lead, -p.lead)
    assert torch.equal(out[live], again[0][live]) and torch.equal(lse[live], again[1][live])


def test_long_contexts_are_split_and_joined():
    """Records of many workgroups to a unit, and of units that begin inside one."""
    Problem([9000], [3], (2, 1), page=64, seed=9).check()
    Problem([20000, 5, 3000], [2, 5, 9], (4, 1), page=64, seed=10).check(torch.bfloat16)
    Problem([4000], [70], (2, 1), page=64, seed=11, tree=False).check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_units_than_workgroups(dtype):
    """Parts of the line that begin inside a unit and go on behind it (wide row tiles
    put that rest off), and whole units between."""
    held = [20 + 37 * b % 400 for b in range(70)]
    Problem(held, [2] * 70, (264, 8), tree=dtype is torch.float32, seed=27).check(dtype)


def test_masks_that_leave_rows_empty():
    """No context and no bits; and bits that no node, word or row has."""
    p = Problem([0, 0, 40], [6, 3, 5], (4, 2), seed=12)
    p.mask[p.lead: p.lead + 4] = 0
    p.mask[p.lead + 9:] = 0
    p.check()
    p.check(torch.bfloat16)
    full = Problem([0, 9], [6, 70], (4, 2), seed=13, words=1)          # nodes past 64 are not seen
    full.mask[full.lead: full.lead + 6] = -1
    full.check()
    wide = Problem([20], [70], (4, 2), seed=14, words=5)
    wide.mask[:, 2:] = -1
    wide.check()


def test_what_is_hidden_has_no_influence():
    """NaN and infinities in keys and values of hidden nodes and unused slots."""
    for heads, new in (((4, 2), 12), ((16, 1), 30)):
        for k_bad, v_bad in ((math.nan, math.nan), (math.inf, math.inf), (0.0, -math.inf), (3.0e38, math.nan)):
            p = Problem([50], [new], heads, seed=15)
            clean = p.run(torch.float32)
            # node new - 1 and node 3 are hidden from all but themselves
            for j in (3, new - 1):
                others = torch.tensor([i for i in range(new) if i != j]) + p.lead
                p.mask[others] &= ~(1 << j)
                p.mask[p.lead + j] |= 1 << j
            clean = p.run(torch.float32)
            cache = p.cache.to(DEV)
            for j in (3, new - 1):
                t = 50 + j
                cache.k[cache.table[0, t // 16].long(), :, t % 16] = k_bad
                cache.v[cache.table[0, t // 16].long(), :, t % 16] = v_bad
            out, lse = p.run(torch.float32, cache=cache)
            see = torch.tensor([i for i in range(new) if i not in (3, new - 1)]) + p.lead
            assert torch.equal(out[see], clean[0][see]) and torch.equal(lse[see], clean[1][see])
            for j in (3, new - 1):
                assert bool(torch.isfinite(lse[p.lead + j]).all()) == (k_bad in (0.0,)) or k_bad == 3.0e38
                if k_bad == 0.0:       # a weight that is not 0 times the value
                    assert bool((out[p.lead + j] == v_bad).all())


def test_a_value_of_the_context_reaches_all():
    p = Problem([50], [8], (4, 2), seed=16)
    cache = p.cache.to(DEV)
    cache.v[cache.table[0, 0].long(), :, 5, 7] = math.inf
    out, _ = p.run(torch.float32, cache=cache)
    live = out[p.lead: -p.lead]
    assert bool((live[..., 7] == math.inf).all()) and bool(torch.isfinite(live[..., :7]).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("extra", [0, LONG])
@pytest.mark.parametrize("held, new, heads", [(300, 5, (4, 2)), (700, 30, (2, 1)), (1500, 40, (8, 1)), (9000, 3, (2, 1))], ids=str)
def test_infinities_that_are_seen(held, new, heads, extra, dtype):
    """Infinities and NaN in the context, far from the nodes and near: their dims are
    infinite or NaN in every row, the other dims as the definition has them."""
    p = Problem([held], [new], heads, seed=25, extra_width=extra)
    odd = {7: (3, math.inf), 64: (held // 2, -math.inf), 65: (held - 1, math.nan), 127: (held // 3, math.inf)}
    cache = p.cache.to(DEV)
    for dim, (t, x) in odd.items():
        p.cache.v[p.cache.table[0, t // 16].long(), :, t % 16, dim] = 0
        cache.v[cache.table[0, t // 16].long(), :, t % 16, dim] = x
    # both signs in one dim
    for t, x in ((5, math.inf), (held - 2, -math.inf)):
        p.cache.v[p.cache.table[0, t // 16].long(), :, t % 16, 100] = 0
        cache.v[cache.table[0, t // 16].long(), :, t % 16, 100] = x
    out, lse = (x.double().cpu()[p.lead: -p.lead] for x in p.run(dtype, cache=cache))
    for dim, (_, x) in odd.items():
        assert bool((out[..., dim].isnan() if math.isnan(x) else out[..., dim] == x).all()), dim
    assert bool(out[..., 100].isnan().all())
    ref = R.attend(p.q, p.cache.k, p.cache.v, p.cache.table, p.context, p.offsets, p.mask, p.scale)
    far, far_lse = (x[p.lead: -p.lead] for x in R.attend_bounds(*ref, dtype is torch.bfloat16))
    plain = [d for d in range(128) if d not in odd and d != 100]
    assert bool(((out - ref[0][p.lead: -p.lead]).abs() <= far)[..., plain].all())
    assert bool(((lse - ref[1][p.lead: -p.lead]).abs() <= far_lse).all())


@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0, 1e-30])
def test_scales(scale):
    p = Problem([300], [9], (4, 2), seed=17)
    p.scale = scale
    p.check()
    p.check(torch.bfloat16)


def test_sharp_and_growing_scores():
    """Scores that grow along the context move the reference again and again."""
    p = Problem([600], [6], (4, 1), seed=18, sharp=6.0)
    t = torch.arange(606)
    pages = p.cache.table[0][t // 16].long()
    u = p.q[p.lead, 0].float()
    p.cache.k[pages, :, t % 16] += (u * (t[:, None] / 606.0) ** 2).bfloat16()[:, None]
    p.check()
    p.check(torch.bfloat16)


def test_large_values():
    p = Problem([200], [5], (4, 1), seed=19)
    big = 2.0 ** 110
    p.cache.v.copy_((p.cache.v.float() * big).bfloat16())
    p.check()


def test_passed_over_sequences_and_bad_pages():
    p = Problem([30, 40, 50], [4, 4, 4], (4, 2), seed=20)
    p.context = torch.tensor([-1, 40, 61], dtype=torch.int32)     # unused; as it is; does not fit (4 pages)
    p.check()
    q = Problem([300], [4], (4, 2), seed=21)
    cache = q.cache.to(DEV)
    cache.table[0, 3], cache.table[0, 5] = 10 ** 6, -7             # clamped: unspecified, but read inside the pools
    q.run(torch.float32, cache=cache)
    for bad in ([0, 50], [-9, 4], [4, 2], [2 ** 31 - 1, -2 ** 31]):
        q.offsets = torch.tensor(bad, dtype=torch.int32)
        q.run(torch.float32)
    torch.cuda.synchronize()


def test_same_bits_every_time():
    p = Problem([3000, 100, 0, 777], [16, 3, 9, 1], (8, 2), seed=22)
    cache = p.cache.to(DEV)
    for dtype in DTYPES:
        first = p.run(dtype, cache=cache)
        ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device=DEV)
        for kw in ({}, {"workspace": ws}, {"workspace": ws}):
            again = p.run(dtype, cache=cache, **kw)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_chain_equals_its_mask_and_single_tokens_decode():
    """Without a mask as with the mask of a chain; and one node at a time as the
    decode call over the same cache."""
    p = Problem([400, 33], [7, 7], (8, 2), tree=False, seed=23, offsets=None)
    plain = p.run(torch.float32)
    p.mask = torch.tensor([R.bits(range(i + 1), 1) for _ in range(2) for i in range(7)], dtype=torch.int64)
    masked = p.run(torch.float32)
    assert torch.equal(plain[0], masked[0]) and torch.equal(plain[1], masked[1])
    c = p.cache.to(DEV)
    for i in range(7):
        out, lse, _ = api.decode_attention(p.q.view(2, 7, 8, 128)[:, i].contiguous().to(DEV), c.k, c.v, c.table.clamp_min(0),
                                           (p.context + i + 1).to(DEV), block_size=64, tau=0.0, phi=0.0, patience=1,
                                           no_detector=True)
        # both keep fp32 throughout
        assert float((out - plain[0].view(2, 7, 8, 128)[:, i]).abs().max()) < 2e-5
        assert float((lse - plain[1].view(2, 7, 8)[:, i]).abs().max()) < 2e-5


def test_graphs_streams_and_a_shared_workspace():
    p = Problem([900, 64], [5, 9], (8, 2), seed=24)
    c = p.cache.to(DEV)
    q, context, mask, offsets = (x.to(DEV) for x in (p.q, p.context, p.mask, p.offsets))
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = api.tree_attention(q, c.k, c.v, c.table, context, mask=mask, token_offsets=offsets)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(api.tree_attention(q, c.k, c.v, c.table, context, mask=mask, token_offsets=offsets))
        graphs.append(g)
    for step in range(3):
        q.copy_(torch.randn(q.shape, generator=p.gen).bfloat16())
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graphs[1].replay()
        graphs[0].replay()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        eager = api.tree_attention(q, c.k, c.v, c.table, context, mask=mask, token_offsets=offsets)
        live = slice(p.lead, -p.lead)
        for out, lse in outs:
            assert torch.equal(out[live], eager[0][live]) and torch.equal(lse[live], eager[1][live])


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    """Batches, heads, pages, contexts and masks at random, every row tile's height
    among them; bits of the masks at random too, not only trees."""
    gen = torch.Generator().manual_seed(1000 + seed)
    pick = lambda *xs: xs[int(torch.randint(0, len(xs), (1,), generator=gen))]  # noqa: E731
    number = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=gen))  # noqa: E731
    H, g = pick((1, 1), (2, 3), (1, 7), (4, 2), (1, 16), (2, 5), (1, 33), (1, 100))
    B = pick(1, 2, 5, 13)
    top = pick(20, 300, 1500 if B < 5 else 200)
    nodes = max(1, pick(3, 30, 150) // (1 + g * B // 20))
    held, new = [number(0, top) for _ in range(B)], [number(0, nodes) for _ in range(B)]
    new[0] = max(new[0], 1)
    p = Problem(held, new, (H * g, H), page=pick(16, 32, 128), tree=pick(True, False), seed=seed, pad=pick(0, 1),
                sharp=pick(0.3, 1.0, 4.0), extra_width=pick(0, LONG))
    if p.mask is not None and pick(True, False):
        p.mask = torch.randint(-2 ** 63, 2 ** 63 - 1, p.mask.shape, generator=gen)
    p.scale = pick(1 / math.sqrt(128), -0.05, 0.2)
    p.check(pick(*DTYPES))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("batch,nodes,group", [(256, 1, 8), (512, 8, 8), (512, 16, 8)])
def test_small_probabilities_behind_large_ones(batch, nodes, group, dtype):
    """128 tokens of weight 1 come first, and 16K of 2^-20.5, each of them below half
    a step of a sum that holds the first ones (16 of them or more): together they are
    8.6e-5 of it.  Scores are exact: 0 and -16 * 8.  A sum may add a tile's part at a
    time, of 32 tokens or more, and within it up to 16, each addition and the few that
    join the parts off by 2^-24 of the sum, and the logarithm is off by two steps."""
    context, page, scale = 16384, 128, 0.1109375
    pages = context // page + 1
    k = torch.zeros(pages, 1, page, 128, dtype=torch.bfloat16, device=DEV)
    k[1:, :, :, 0] = -8.0
    v = torch.ones_like(k)
    q = torch.zeros(batch * nodes, group, 128, dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = 16.0
    table = torch.arange(pages, dtype=torch.int32, device=DEV).expand(batch, pages).contiguous()
    held = torch.full((batch,), context, dtype=torch.int32, device=DEV)
    _, lse = api.tree_attention(q, k, v, table, held, softmax_scale=scale, out_dtype=dtype)
    small = context - 128 + 1 + torch.arange(nodes, dtype=torch.float64)
    ref = torch.log(128 + small * math.exp(-128 * scale))
    tol = (context / 32 + 24) * 2.0 ** -24 + 2 * 5 * 2.0 ** -23
    err = (lse.cpu().double().view(batch, nodes, group) - ref[:, None]).abs().max().item()
    assert err <= tol, (err, tol)
