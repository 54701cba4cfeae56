"""Trees' masks, verification of drafts and the move of accepted tokens against
their definitions (needs a gfx950 GPU).  Results are whole numbers or copies: equal."""
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


def _dev(t):
    return None if t is None else t.to(DEV)


@pytest.mark.parametrize("new", [[1], [5], [64], [65, 3, 0, 130], [1024], [2] * 300], ids=str)
@pytest.mark.parametrize("words", [1, 3, 16])
def test_layout(new, words):
    gen = torch.Generator().manual_seed(sum(new) + words)
    parents = [R.random_parents(gen, n, chain=i % 3 == 2) for i, n in enumerate(new)]
    held = torch.randint(0, 100000, (len(new),), generator=gen).int()
    offsets = torch.tensor([sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32)
    flat = torch.tensor(sum(parents, []), dtype=torch.int32)
    mask, positions = api.tree_layout(flat.to(DEV), held.to(DEV), mask_words=words, token_offsets=offsets.to(DEV))
    want = [R.bits(R.ancestors(p, i), words) for p in parents for i in range(len(p))]
    depth = [int(held[b]) + len(R.ancestors(p, i)) - 1 for b, p in enumerate(parents) for i in range(len(p))]
    assert mask.tolist() == want and positions.tolist() == depth


def test_layout_of_odd_parents():
    """A parent that is no earlier node ends the walk; equal lengths need no offsets;
    a sequence with a negative context, or of too many nodes, is passed over."""
    parents = torch.tensor([-1, 5, 0, 2, -9, 4, 6, 6], dtype=torch.int32, device=DEV)
    mask, positions = api.tree_layout(parents, torch.tensor([10, 20], dtype=torch.int32, device=DEV))
    # the second sequence: nodes 0 (parent -9), 1 (parent 4, later), 2 and 3 (parent 6, later)
    assert mask[:, 0].tolist() == [1, 2, 5, 13, 1, 2, 4, 8] and positions.tolist() == [10, 10, 11, 12, 20, 20, 20, 20]
    flat = torch.zeros(1030, dtype=torch.int32, device=DEV)
    out = torch.full((1030, 1), 9, dtype=torch.int64, device=DEV)
    offsets = torch.tensor([0, 2, 4, 1030], dtype=torch.int32, device=DEV)
    context = torch.tensor([-1, 3, 0], dtype=torch.int32, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    assert _lib.tree_layout(3, 1030, flat.data_ptr(), offsets.data_ptr(), context.data_ptr(), 1, out.data_ptr(), 0, stream) == 0
    assert out[:5, 0].tolist() == [9, 9, 1, 3, 9] and bool((out[4:] == 9).all())


def _drafts(gen, new, V, *, chain, sampled, dtype, sharp=2.0, near=0.5):
    rows = sum(new)
    target = torch.softmax(sharp * torch.randn(rows, V, generator=gen), -1)
    guess = torch.softmax(target.log() + near * torch.randn(rows, V, generator=gen), -1)
    parents, tokens, at = [], [], 0
    for n in new:
        p = R.random_parents(gen, n, chain)
        nth = {}
        for i in range(n):
            if i == 0:
                tokens.append(0)
                continue
            row = guess[at + p[i]]
            if sampled:
                tokens.append(int(torch.multinomial(row.to(dtype).float(), 1, generator=gen)))
            else:
                k = nth.get(p[i], 0)
                nth[p[i]] = k + 1
                tokens.append(int(row.argsort(descending=True)[min(k, V - 1)]))
        parents += p
        at += n
    as_int = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return (target.to(dtype), guess.to(dtype) if sampled else None, as_int(tokens), as_int(parents),
            torch.rand(rows, generator=gen), torch.rand(len(new), generator=gen),
            as_int([sum(new[:b]) for b in range(len(new) + 1)]))


def _compare(args, max_path):
    target, draft, tokens, parents, uniforms, last, offsets = args
    got = api.verify_drafts(_dev(target), _dev(tokens), _dev(parents), _dev(uniforms), _dev(last), draft=_dev(draft),
                            token_offsets=_dev(offsets), max_path=max_path)
    want = R.verify_all(target, draft, tokens, parents, uniforms, last, offsets, max_path)
    for name, a, b in zip(("accepted", "counts", "next"), got, want):
        assert a.cpu().tolist() == b.tolist(), name
    return want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("chain", [True, False])
@pytest.mark.parametrize("V", [2, 63, 1000, 5003])
def test_verify(V, chain, sampled, dtype):
    gen = torch.Generator().manual_seed(V + 2 * chain + sampled)
    seen = 0
    for new in ([1], [2], [9] * 12, [1, 30, 0, 70, 5, 16]):
        want = _compare(_drafts(gen, new, V, chain=chain, sampled=sampled, dtype=dtype), max_path=max(new))
        seen += int((want[1] > 1).sum())
    assert seen > 0                      # drafts have been accepted


def test_verify_of_many_sequences_and_large_vocabularies():
    gen = torch.Generator().manual_seed(1)
    _compare(_drafts(gen, [3] * 700, 300, chain=False, sampled=True, dtype=torch.float32), max_path=3)
    for sampled in (True, False):
        _compare(_drafts(gen, [6, 12, 4], 151001, chain=False, sampled=sampled, dtype=torch.float32, sharp=4.0), max_path=12)
    _compare(_drafts(gen, [1024, 5], 40, chain=False, sampled=True, dtype=torch.float32), max_path=1024)
    _compare(_drafts(gen, [1024, 5], 40, chain=False, sampled=False, dtype=torch.float32), max_path=1024)
    _compare(_drafts(gen, [1025, 5], 10, chain=True, sampled=False, dtype=torch.float32), max_path=30)


def test_verify_many_rejected_siblings():
    """Twelve children of node 0 whose tokens the target does not have: a sum over the
    vocabulary for each."""
    gen = torch.Generator().manual_seed(2)
    V, n = 3001, 13
    target, draft = torch.zeros(n, V), torch.zeros(n, V)
    target[:, : V // 2] = torch.rand(n, V // 2, generator=gen)
    draft[:, V // 4:] = torch.rand(n, V - V // 4, generator=gen)
    target, draft = target / target.sum(-1, keepdim=True), draft / draft.sum(-1, keepdim=True)
    tokens = torch.randint(V // 2, V, (n,), generator=gen).int()
    tokens[n - 1] = V // 3
    parents = torch.tensor([-1] + [0] * (n - 1), dtype=torch.int32)
    for _ in range(5):
        args = (target, draft, tokens, parents, torch.rand(n, generator=gen), torch.rand(1, generator=gen),
                torch.tensor([0, n], dtype=torch.int32))
        _compare(args, 4)


def test_greedy_by_one_hot_rows():
    gen = torch.Generator().manual_seed(3)
    V, n = 500, 20
    best = torch.randint(0, V, (n,), generator=gen)
    target = torch.nn.functional.one_hot(best, V).float()
    parents = torch.tensor(R.random_parents(gen, n), dtype=torch.int32)
    tokens = torch.randint(0, V, (n,), generator=gen).int()
    path = [0]
    for c in range(1, n):                       # the right token on a path of first children
        if parents[c] == path[-1] and len(path) < 4:
            tokens[c] = best[path[-1]]
            path.append(c)
    accepted, counts, following = api.verify_drafts(
        target.to(DEV), tokens.to(DEV), parents.to(DEV), torch.rand(n, generator=gen).to(DEV), torch.rand(1, generator=gen).to(DEV))
    assert accepted[0, : len(path)].tolist() == path
    at = int(accepted[0, int(counts[0]) - 1])
    assert int(following[0]) == int(best[at])


def test_verify_edges():
    """Equal tokens among siblings, tokens outside the vocabulary, paths cut short,
    rows that p and q share, random numbers of 0 and almost 1, strided rows."""
    V = 64
    gen = torch.Generator().manual_seed(4)
    p = torch.softmax(torch.randn(8, V, generator=gen), -1)
    off = torch.tensor([0, 8], dtype=torch.int32)
    parents = torch.tensor([-1, 0, 0, 0, 0, 1, 2, 5], dtype=torch.int32)
    tokens = torch.tensor([0, 5, 5, -1, V, 7, 9, 9], dtype=torch.int32)
    top = 1 - 2.0 ** -24
    for u in (0.0, 0.5, top):
        for last in (0.0, 0.3, top):
            for draft in (None, p, torch.softmax(torch.randn(8, V, generator=gen), -1)):
                for max_path in (1, 2, 8):
                    _compare((p, draft, tokens, parents, torch.full((8,), u), torch.tensor([last]), off), max_path)
    # nothing left: all mass on rejected tokens, or p within q
    one = torch.zeros(8, V)
    one[:, 5] = 0.5
    _compare((one, None, tokens, parents, torch.full((8,), top), torch.tensor([0.5]), off), 8)
    _compare((one, one * 2, tokens, parents, torch.full((8,), top), torch.tensor([0.5]), off), 8)
    # rows with a stride, in an odd place
    wide = torch.rand(8, V + 3, generator=gen)
    got = api.verify_drafts(wide.to(DEV)[:, 1: V + 1], tokens.to(DEV), parents.to(DEV), torch.full((8,), 0.5, device=DEV),
                            torch.tensor([0.7], device=DEV), draft=p.to(DEV))
    want = R.verify_all(wide[:, 1: V + 1], p, tokens, parents, torch.full((8,), 0.5), torch.tensor([0.7]), None, 8)
    for a, b in zip(got, want):
        assert a.cpu().tolist() == b.tolist()


def test_verify_of_nan_gives_some_token():
    V = 5000
    p = torch.rand(4, V)
    p[:, 77] = math.nan
    parents, tokens = torch.tensor([-1, 0, 1, 0]).int().to(DEV), torch.tensor([0, 77, 3, 4]).int().to(DEV)
    for draft in (None, p.to(DEV), torch.rand(4, V, device=DEV)):
        _, counts, following = api.verify_drafts(p.to(DEV), tokens, parents, torch.full((4,), 0.9, device=DEV),
                                                 torch.tensor([0.5], device=DEV), draft=draft)
        assert 1 <= int(counts[0]) <= 4 and 0 <= int(following[0]) < V


def test_accepted_tokens_have_the_targets_distribution():
    """40000 sequences with a chain of one draft over a vocabulary of 6: the first
    token that follows node 0 against the target, within 5 standard deviations."""
    gen = torch.Generator().manual_seed(5)
    B, V = 40000, 6
    p, q = torch.tensor([0.4, 0.3, 0.15, 0.1, 0.05, 0.0]), torch.tensor([0.1, 0.2, 0.4, 0.05, 0.05, 0.2])
    drawn = torch.multinomial(q.expand(B, V), 1, generator=gen)[:, 0].int()
    tokens = torch.stack([torch.zeros(B, dtype=torch.int32), drawn], 1).reshape(-1)
    parents = torch.tensor([-1, 0], dtype=torch.int32).repeat(B)
    accepted, counts, following = (x.cpu() for x in api.verify_drafts(
        p.expand(2 * B, V).contiguous().to(DEV), tokens.to(DEV), parents.to(DEV), torch.rand(2 * B, generator=gen).to(DEV),
        torch.rand(B, generator=gen).to(DEV), draft=q.expand(2 * B, V).contiguous().to(DEV)))
    first = torch.where(counts == 2, drawn, following)
    share = torch.bincount(first.long(), minlength=V).double() / B
    assert bool(((share - p).abs() <= 5 * (p * (1 - p) / B).sqrt() + 1e-9).all())


@pytest.mark.parametrize("page, heads, pad", [(16, 2, 0), (64, 8, 1), (32, 1, 0)])
def test_keep(page, heads, pad):
    gen = torch.Generator().manual_seed(page)
    held, new, paths = [0, 17, 130, 63, 5], [12, 5, 60, 9, 1], [[0, 2, 3, 7, 11], [0], [0, 5, 6, 20, 21, 22, 59], [3, 8], [0]]
    cpu = R.Cache(gen, [a + b for a, b in zip(held, new)], heads, page, pad=pad)
    cache = cpu.to(DEV)
    width = 9
    accepted = torch.tensor([p + [-1] * (width - len(p)) for p in paths], dtype=torch.int32)
    counts = torch.tensor([len(p) for p in paths], dtype=torch.int32)
    api.keep_accepted(cache.k, cache.v, cache.table, torch.tensor(held, dtype=torch.int32, device=DEV), accepted.to(DEV), counts.to(DEV))
    for name in ("k", "v"):
        was, want = getattr(cpu, name), getattr(cpu, name).clone()
        for b, p in enumerate(paths):
            for j, node in enumerate(p):
                a, c = held[b] + node, held[b] + j
                want[cpu.table[b, c // page].long(), :, c % page] = was[cpu.table[b, a // page].long(), :, a % page]
        assert torch.equal(getattr(cache, name).cpu().nan_to_num(123), want.nan_to_num(123))


def test_keep_passes_over_lists_that_are_none():
    gen = torch.Generator().manual_seed(7)
    cpu = R.Cache(gen, [32] * 7, 2, 16)
    cpu.table[6, 1] = -1
    cache = cpu.to(DEV)
    accepted = torch.tensor([[0, 2, 2], [2, 1, 3], [-1, 4, 5], [0, 5, 40], [0, 5, 9], [1, 2, 3], [0, 20, 25]], dtype=torch.int32, device=DEV)
    counts = torch.tensor([3, 3, 3, 3, 4, 3, 3], dtype=torch.int32, device=DEV)
    context = torch.tensor([0, 0, 0, 0, 0, -1, 0], dtype=torch.int32, device=DEV)
    api.keep_accepted(cache.k, cache.v, cache.table, context, accepted, counts)
    assert torch.equal(cache.k.cpu().nan_to_num(123), cpu.k.nan_to_num(123))
    assert torch.equal(cache.v.cpu().nan_to_num(123), cpu.v.nan_to_num(123))
