"""The calls on drafted tokens in a row, as a decode step uses them, over several
steps against the same steps in 64 bits (needs a gfx950 GPU)."""
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


@pytest.mark.parametrize("captured", [False, True])
def test_steps(captured):
    """Three sequences (and an unused one) take four steps of ragged trees.  After every
    step the cache holds what an append of the accepted tokens alone, at their own
    positions, would have left, and attention over it agrees with the definition."""
    gen = torch.Generator().manual_seed(1)
    Hq, H, page, V, B = 8, 2, 16, 300, 4
    width = 8
    pools = [torch.zeros((B * width, H, page, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    table = torch.randperm(B * width, generator=gen).int().view(B, width).to(DEV)
    rope = api.rope_frequencies(128, base=5e5, factor=2.0, original_len=64)
    rows = 24
    state = dict(q=torch.empty(rows, Hq, 128), k=torch.empty(rows, H, 128), v=torch.empty(rows, H, 128),
                 target=torch.empty(rows, V), uniforms=torch.empty(rows), last=torch.empty(B))
    state = {n: t.to(DEV, torch.bfloat16 if n in "qkv" else torch.float32) for n, t in state.items()}
    ints = dict(parents=torch.zeros(rows), tokens=torch.zeros(rows), offsets=torch.zeros(B + 1), context=torch.zeros(B))
    ints = {n: t.int().to(DEV) for n, t in ints.items()}

    def step():
        mask, positions = api.tree_layout(ints["parents"], ints["context"], token_offsets=ints["offsets"])
        q = api.rope_append(*pools, state["k"], state["v"], table, ints["context"], rope=rope, q=state["q"],
                            token_offsets=ints["offsets"], row_positions=positions)
        out, lse = api.tree_attention(q, *pools, table, ints["context"], mask=mask, token_offsets=ints["offsets"])
        accepted, counts, following = api.verify_drafts(state["target"], ints["tokens"], ints["parents"], state["uniforms"],
                                                        state["last"], token_offsets=ints["offsets"], max_path=6)
        api.keep_accepted(*pools, table, ints["context"], accepted, counts)
        return mask, positions, q, out, lse, accepted, counts, following

    graph = None
    kept = [[] for _ in range(B)]                       # rotated key and value of every token, by sequence
    held = [0, 0, 0, -1]
    for turn in range(4):
        new = [[9, 5, 3, 4], [1, 8, 6, 4], [12, 1, 4, 2], [7, 7, 7, 1]][turn]
        parents = sum((R.random_parents(gen, n) for n in new), [])
        parents += [0] * (rows - len(parents))
        for n in "qkv":
            state[n].copy_(torch.randn(state[n].shape, generator=gen))
        target = torch.softmax(2 * torch.randn(rows, V, generator=gen), -1)
        first = [sum(new[:b]) for b in range(B + 1)]
        tokens = torch.zeros(rows, dtype=torch.int32)
        for b, n in enumerate(new):
            for i in range(1, n):
                tokens[first[b] + i] = int(target[first[b] + parents[first[b] + i]].argmax())
        state["target"].copy_(target)
        state["uniforms"].copy_(torch.rand(rows, generator=gen) * 0.2)
        state["last"].copy_(torch.rand(B, generator=gen))
        for n, x in (("parents", parents), ("tokens", tokens), ("offsets", first), ("context", held)):
            ints[n].copy_(torch.as_tensor(x, dtype=torch.int32))
        before = [p.clone() for p in pools]
        if captured and graph is None:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()                                  # warm, then as it was
            torch.cuda.current_stream().wait_stream(side)
            for p, was in zip(pools, before):
                p.copy_(was)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                results = step()
        if captured:
            graph.replay()
        else:
            results = step()
        torch.cuda.synchronize()
        mask, positions, q, out, lse, accepted, counts, following = (x.cpu() for x in results)
        # attention ran over the cache as the append left it: rebuild that, from the kept
        # tokens and this step's nodes
        k_pool, v_pool = (torch.zeros(B * width, H, page, 128, dtype=torch.bfloat16) for _ in range(2))
        for b, n in enumerate(new[:3]):
            span = slice(first[b], first[b] + n)
            depth = torch.tensor([len(R.ancestors(parents[span], i)) - 1 for i in range(n)])
            assert positions[span].tolist() == (held[b] + depth).tolist()
            turned, size = R.rotate(state["k"][span].cpu(), held[b] + depth, rope.freqs.cpu(), "half", rope.scale)
            q_ref, q_size = R.rotate(state["q"][span].cpu(), held[b] + depth, rope.freqs.cpu(), "half", rope.scale)
            assert bool(((q[span].double() - q_ref).abs() <= 2.0 ** -8 * (q_ref.abs() + 2.0 ** -20) + q_size * 2.0 ** -20).all())
            nodes = api.rope_rows(state["k"][span].contiguous(), positions[span].to(DEV), rope).cpu()
            assert bool(((nodes.double() - turned).abs() <= 2.0 ** -8 * (turned.abs() + 2.0 ** -20) + size * 2.0 ** -20).all())
            every = kept[b] + [(nodes[i], state["v"][first[b] + i].cpu()) for i in range(n)]
            for t, (key, value) in enumerate(every):
                where = int(table[b, t // page]), slice(None), t % page
                k_pool[where], v_pool[where] = key, value
            lines = [R.bits(R.ancestors(parents[span], i), 1) for i in range(n)]
            assert mask[span].tolist() == lines
        live = slice(0, first[3])
        ref = R.attend(q[live], k_pool, v_pool, table.cpu()[:3], torch.tensor(held[:3]), torch.tensor(first[:4]), mask[live],
                       1 / math.sqrt(128))
        far, far_lse = R.attend_bounds(*ref, False)
        assert bool(((out[live].double() - ref[0]).abs() <= far).all()) and bool(((lse[live].double() - ref[1]).abs() <= far_lse).all())
        want = R.verify_all(target, None, tokens, torch.tensor(parents), state["uniforms"].cpu(), state["last"].cpu(), first, 6)
        assert accepted.tolist() == want[0].tolist() and counts.tolist() == want[1].tolist() and following.tolist() == want[2].tolist()
        for b in range(3):
            n = int(counts[b])
            for j in range(n):
                node = int(accepted[b, j])
                assert int(positions[first[b] + node]) == held[b] + j
                slot = held[b] + node
                kept[b].append((k_pool[int(table[b, slot // page]), :, slot % page].clone(),
                                v_pool[int(table[b, slot // page]), :, slot % page].clone()))
            held[b] += n
            for t, (key, value) in enumerate(kept[b]):
                where = int(table[b, t // page]), slice(None), t % page
                assert torch.equal(pools[0][where].cpu(), key) and torch.equal(pools[1][where].cpu(), value)
    assert max(held) > 6


def test_far_offsets():
    """Pages 2^28 elements apart: bytes and elements pass 32 bits."""
    gen = torch.Generator().manual_seed(2)
    H, page, n, held = 2, 16, 5, 40
    near = R.Cache(gen, [held + n], H, page, spare=6)
    pages, stride = near.k.shape[0], 1 << 28
    far = object.__new__(R.Cache)
    for name in ("k", "v"):
        base = torch.empty((pages - 1) * stride + H * page * 128, dtype=torch.bfloat16, device=DEV)
        setattr(far, name, base.as_strided(near.k.shape, (stride, page * 128, 128, 1)))
        getattr(far, name).copy_(getattr(near, name))
    near, far.table = near.to(DEV), near.table.to(DEV)
    context = torch.tensor([held], dtype=torch.int32, device=DEV)
    x = torch.randn(n, H, 128, generator=gen).bfloat16().to(DEV)
    q = torch.randn(n, 4, 128, generator=gen).bfloat16().to(DEV)
    rope = api.rope_frequencies(128)
    accepted, counts = torch.tensor([[0, 2, 4]], dtype=torch.int32, device=DEV), torch.tensor([3], dtype=torch.int32, device=DEV)
    results = []
    for c in (near, far):
        turned = api.rope_append(c.k, c.v, x, x, c.table, context, rope=rope, q=q)
        out, lse = api.tree_attention(turned, c.k, c.v, c.table, context)
        api.keep_accepted(c.k, c.v, c.table, context, accepted, counts)
        results.append((turned, out, lse, c.k.contiguous().view(torch.int16), c.v.contiguous().view(torch.int16)))
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_nothing_to_do():
    """No rows, no sequences, sequences without nodes."""
    c = R.Cache(torch.Generator().manual_seed(3), [20], 2, 16).to(DEV)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    one, offsets = torch.tensor([4], dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    rows, q = torch.zeros(0, 2, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(0, 4, 128, dtype=torch.bfloat16, device=DEV)
    was = c.k.clone().view(torch.int16)
    for kw in ({}, {"token_offsets": offsets}):
        assert api.rope_append(c.k, c.v, rows, rows, c.table, one, q=q, **kw).shape == (0, 4, 128)
        assert api.tree_attention(q, c.k, c.v, c.table, one, **kw)[0].shape == (0, 4, 128)
        assert api.tree_layout(none, one, **kw)[0].shape == (0, 1)
        accepted, counts, following = api.verify_drafts(
            torch.zeros(0, 10, device=DEV), none, none, torch.zeros(0, device=DEV), torch.zeros(1, device=DEV), max_path=2, **kw)
        assert accepted.tolist() == [[-1, -1]] and counts.tolist() == [0] and following.tolist() == [-1]
        api.keep_accepted(c.k, c.v, c.table, one, accepted, counts)
    assert api.rope_rows(rows, none, api.rope_frequencies(64)).shape == (0, 2, 128)
    assert torch.equal(c.k.view(torch.int16), was)
    with pytest.raises(ValueError):
        api.tree_attention(q, c.k, c.v, c.table, one, mask=torch.zeros(0, 0, dtype=torch.int64, device=DEV))
