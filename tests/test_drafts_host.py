"""Refusals of the calls on drafted tokens, before anything is launched (no GPU),
the plain references of the GPU tests, and the frequencies of rotary positions."""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

import draftref as R
from paper_2606_00024_amd import _lib, api

PTR = 4096      # never read: every call here is refused, or has nothing to do
OK, BAD, NO, SMALL = _lib.OK, _lib.ERR_INVALID_ARG, _lib.ERR_UNSUPPORTED, _lib.ERR_WORKSPACE_TOO_SMALL


def _shape(**kw):
    d = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, block_size=64, page_size=64,
             num_pages=40, max_pages_per_seq=16, max_blocks_per_list=0, list_per_head=1,
             k_stride_page=2 * 64 * 128, k_stride_head=64 * 128, k_stride_token=128,
             v_stride_page=2 * 64 * 128, v_stride_head=64 * 128, v_stride_token=128)
    d.update(kw)
    return _lib.DecodeShape(**d)


def _rows(heads=2, **kw):
    d = dict(dtype=_lib.ROWS_BF16, heads=heads, stride_row=heads * 128, stride_head=128)
    d.update(kw)
    return _lib.Rows(**d)


def _rope(**kw):
    d = dict(layout=_lib.ROPE_HALF, rot_dim=128, scale=1.0)
    d.update(kw)
    return _lib.RopeSpec(**d)


def _rope_rows(rope=None, rows=4, x_rows=None, out_rows=None, **kw):
    a = dict(x=PTR, out=PTR, positions=PTR, freqs=PTR)
    a.update(kw)
    return _lib.rope_rows(rope or _rope(), rows, x_rows or _rows(), a["x"], out_rows or _rows(), a["out"],
                          a["positions"], a["freqs"], 0)


def _append(shape=None, rope="usual", rows=4, q_rows=None, q_out_rows=None, k_rows=None, v_rows=None, **kw):
    a = dict(q=0, q_out=0, k=PTR, v=PTR, row_offsets=0, context_lens=PTR, row_positions=0, freqs=PTR,
             page_table=PTR, k_cache=PTR, v_cache=PTR)
    a.update(kw)
    return _lib.rope_append(shape or _shape(), _rope() if rope == "usual" else rope, rows, q_rows, a["q"],
                            q_out_rows, a["q_out"], k_rows or _rows(), a["k"], v_rows or _rows(), a["v"],
                            a["row_offsets"], a["context_lens"], a["row_positions"], a["freqs"],
                            a["page_table"], a["k_cache"], a["v_cache"], 0)


def _tree_opts(**kw):
    d = dict(softmax_scale=0.1, out_dtype=0, rows=4, mask_words=1, q_stride_row=1024, q_stride_head=128)
    d.update(kw)
    return _lib.TreeOpts(**d)


def _tree(shape=None, opts=None, **kw):
    a = dict(q=PTR, k=PTR, v=PTR, page_table=PTR, context_lens=PTR, row_offsets=0, mask=PTR, out=PTR, lse=PTR,
             workspace=PTR, workspace_bytes=1 << 30)
    a.update(kw)
    return _lib.tree_attention(shape or _shape(), opts or _tree_opts(), *a.values(), 0)


def _verify_opts(**kw):
    d = dict(batch=2, rows=8, vocab=100, max_path=4, dtype=_lib.ROWS_F32, target_stride=100, draft_stride=100)
    d.update(kw)
    return _lib.VerifyOpts(**d)


def _verify(opts=None, **kw):
    a = dict(target=PTR, draft=PTR, tokens=PTR, parents=PTR, row_offsets=0, uniforms=PTR, last_uniforms=PTR,
             accepted=PTR, counts=PTR, next_tokens=PTR, workspace=PTR, workspace_bytes=1 << 30)
    a.update(kw)
    return _lib.verify_drafts(opts or _verify_opts(), *a.values(), 0)


def _keep(shape=None, max_path=4, **kw):
    a = dict(accepted=PTR, counts=PTR, context_lens=PTR, page_table=PTR, k_cache=PTR, v_cache=PTR)
    a.update(kw)
    return _lib.keep_accepted(shape or _shape(), max_path, *a.values(), 0)


SHAPES = [(dict(num_kv_heads=0), BAD), (dict(batch=-1), BAD), (dict(num_pages=0), BAD), (dict(max_pages_per_seq=0), BAD),
          (dict(k_stride_page=-8), BAD), (dict(head_dim=64, ), NO), (dict(page_size=48), NO), (dict(page_size=8), NO),
          (dict(v_stride_token=132), NO), (dict(k_stride_head=4), NO)]


@pytest.mark.parametrize("bad, status", SHAPES)
def test_caches_that_are_refused(bad, status):
    for call in (_append, _tree, _keep):
        assert call(_shape(**bad)) == status, call


@pytest.mark.parametrize("bad, status", [
    (dict(layout=2), BAD), (dict(rot_dim=-2), BAD), (dict(rot_dim=130), BAD), (dict(rot_dim=31), BAD),
    (dict(scale=math.inf), BAD), (dict(scale=math.nan), BAD)])
def test_rotations_that_are_refused(bad, status):
    assert _rope_rows(_rope(**bad)) == status
    assert _append(rope=_rope(**bad)) == status


@pytest.mark.parametrize("bad, status", [
    (dict(dtype=3), BAD), (dict(dtype=-1), BAD), (dict(heads=0), BAD), (dict(stride_row=-8), BAD),
    (dict(stride_head=-8), BAD), (dict(stride_row=1 << 28), NO), (dict(stride_row=1 << 62), NO),
    (dict(stride_head=1 << 62), NO), (dict(stride_row=260), NO), (dict(stride_head=4), NO),
    (dict(dtype=_lib.ROWS_F32, stride_row=258), NO)])
def test_rows_that_are_refused(bad, status):
    assert _rope_rows(x_rows=_rows(**bad)) == status
    assert _rope_rows(out_rows=_rows(**bad)) == status
    assert _append(k_rows=_rows(**bad)) == status
    assert _append(v_rows=_rows(**bad)) == status


def test_rope_rows_refusals():
    assert _rope_rows(rows=-1) == BAD
    assert _rope_rows(rows=1 << 24) == NO
    assert _rope_rows(out_rows=_rows(3)) == BAD
    for name in ("x", "out", "positions", "freqs"):
        assert _rope_rows(**{name: 0}) == BAD, name
    assert _rope_rows(x=PTR + 8) == NO and _rope_rows(out=PTR + 2) == NO and _rope_rows(freqs=PTR + 4) == BAD
    assert _rope_rows(rows=0, x=0, out=0) == OK


def test_append_refusals():
    q = dict(q=PTR, q_out=PTR, q_rows=_rows(8), q_out_rows=_rows(8))
    assert _append(rows=-1) == BAD and _append(rows=5) == BAD and _append(rows=1 << 24) == NO
    assert _append(k_rows=_rows(3)) == BAD and _append(v_rows=_rows(2, dtype=_lib.ROWS_F16)) == BAD
    assert _append(**{**q, "q_rows": _rows(4)}) == BAD and _append(**{**q, "q_out_rows": _rows(4)}) == BAD
    assert _append(**{**q, "q_rows": _rows(8, dtype=_lib.ROWS_F32)}) == BAD
    assert _append(**{**q, "q_out_rows": _rows(8, dtype=_lib.ROWS_F16)}) == NO
    assert _append(**{**q, "q_out": 0}) == BAD and _append(**{**q, "q_rows": None}) == BAD
    for name in ("k", "v", "context_lens", "freqs", "page_table", "k_cache", "v_cache"):
        assert _append(**{name: 0}) == BAD, name
    for name in ("k", "v", "k_cache", "v_cache"):
        assert _append(**{name: PTR + 8}) == NO, name
    assert _append(rows=0, k=0) == OK and _append(_shape(batch=0), k=0) == OK


def test_layout_refusals():
    call = lambda batch=2, rows=4, parents=PTR, offsets=0, context=PTR, words=1, mask=PTR, positions=PTR: (  # noqa: E731
        _lib.tree_layout(batch, rows, parents, offsets, context, words, mask, positions, 0))
    assert call(batch=-1) == BAD and call(rows=-1) == BAD and call(rows=5) == BAD and call(words=0) == BAD
    assert call(words=17) == NO and call(parents=0) == BAD and call(mask=0) == BAD and call(mask=PTR + 4) == BAD
    assert call(context=0) == BAD
    assert call(rows=2050) == NO and call(rows=0, mask=0) == OK and call(batch=0) == OK


def test_tree_refusals():
    assert _tree(opts=_tree_opts(rows=-1)) == BAD and _tree(opts=_tree_opts(rows=5)) == BAD
    assert _tree(opts=_tree_opts(softmax_scale=math.nan)) == BAD and _tree(opts=_tree_opts(out_dtype=2)) == BAD
    assert _tree(opts=_tree_opts(mask_words=-1)) == BAD and _tree(opts=_tree_opts(mask_words=0)) == BAD
    assert _tree(mask=0) == BAD and _tree(opts=_tree_opts(q_stride_row=-8)) == BAD
    assert _tree(opts=_tree_opts(q_stride_head=4)) == NO and _tree(opts=_tree_opts(rows=1 << 24)) == NO
    assert _tree(_shape(num_q_heads=7)) == BAD and _tree(_shape(num_q_heads=0)) == BAD
    assert _tree(_shape(num_q_heads=258)) == NO
    assert _tree(_shape(max_pages_per_seq=1 << 25)) == NO and _tree(_shape(max_pages_per_seq=(1 << 25) - 1024)) == NO
    for name in ("q", "k", "v", "page_table", "context_lens", "out", "lse"):
        assert _tree(**{name: 0}) == BAD, name
    for name in ("q", "k", "v", "out"):
        assert _tree(**{name: PTR + 8}) == NO, name
    assert _tree(workspace=0) == SMALL and _tree(workspace=PTR + 8) == BAD
    need = _lib.tree_workspace_bytes(_shape(), _tree_opts())
    assert _tree(workspace_bytes=need - 1) == SMALL
    assert _tree(opts=_tree_opts(rows=0), q=0) == OK and _tree(_shape(batch=0), q=0) == OK


def test_tree_workspace_is_a_function_of_shape_and_options():
    sizes = [_lib.tree_workspace_bytes(_shape(batch=b, max_pages_per_seq=w), _tree_opts(rows=r))
             for b, w, r in ((1, 1, 1), (1, 64, 1), (8, 512, 128), (32, 1024, 256), (1, 1024, 16384))]
    assert all(n > 0 for n in sizes) and max(sizes) < 80 << 20
    with pytest.raises(api.ArtError):
        _lib.tree_workspace_bytes(_shape(page_size=24), _tree_opts())


def test_verify_refusals():
    for bad in (dict(batch=-1), dict(rows=-1), dict(rows=7), dict(vocab=0), dict(max_path=0), dict(dtype=3),
                dict(target_stride=99), dict(draft_stride=99)):
        assert _verify(_verify_opts(**bad)) == BAD, bad
    for bad in (dict(vocab=1 << 24, target_stride=1 << 24, draft_stride=1 << 24), dict(rows=1 << 24), dict(batch=1 << 18, rows=0)):
        assert _verify(_verify_opts(**bad)) == NO, bad
    for name in ("target", "tokens", "parents", "uniforms", "last_uniforms", "accepted", "counts", "next_tokens"):
        assert _verify(**{name: 0}) == BAD, name
    assert _verify(target=PTR + 2) == BAD and _verify(draft=PTR + 1) == BAD and _verify(workspace=PTR + 4) == BAD
    assert _verify(_verify_opts(rows=2050)) == NO and _verify(workspace=0) == SMALL
    assert _verify(workspace_bytes=_lib.verify_workspace_bytes(_verify_opts()) - 1) == SMALL
    assert _verify(_verify_opts(batch=0)) == OK


def test_keep_refusals():
    assert _keep(max_path=0) == BAD
    for name in ("accepted", "counts", "context_lens", "page_table", "k_cache", "v_cache"):
        assert _keep(**{name: 0}) == BAD, name
    assert _keep(k_cache=PTR + 8) == NO and _keep(_shape(batch=1 << 20)) == NO
    assert _keep(_shape(batch=0), accepted=0) == OK


def test_tensors_that_are_refused_without_a_gpu():
    pool = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16)
    table, one = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    row = torch.zeros((1, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        api.rope_append(pool, pool, row, row, table, one)
    with pytest.raises(ValueError):
        api.rope_rows(row, one, api.Rope(torch.ones(64, dtype=torch.float64)))
    with pytest.raises(ValueError):
        api.tree_attention(row, pool, pool, table, one)
    with pytest.raises(ValueError):
        api.tree_layout(one, one)
    with pytest.raises(ValueError):
        api.verify_drafts(torch.ones(1, 4), one, one, torch.zeros(1), torch.zeros(1))
    with pytest.raises(ValueError):
        api.keep_accepted(pool, pool, table, one, table, one)


def test_frequencies():
    plain = api.rope_frequencies(64, device="cpu")
    assert plain.scale == 1.0 and plain.freqs.dtype is torch.float64
    assert torch.allclose(plain.freqs, torch.tensor([10000.0 ** (-2 * i / 64) for i in range(32)], dtype=torch.float64), rtol=1e-14)
    longer = api.rope_frequencies(64, factor=4.0, device="cpu")
    assert torch.equal(longer.freqs, plain.freqs / 4) and longer.scale == 1.0
    yarn = api.rope_frequencies(128, base=1e6, factor=4.0, original_len=8192, device="cpu")
    base = api.rope_frequencies(128, base=1e6, device="cpu").freqs
    turns = base * 8192 / (2 * math.pi)
    assert yarn.scale == pytest.approx(0.1 * math.log(4) + 1)
    assert torch.equal(yarn.freqs[turns > 40], base[turns > 40])          # fast pairs stay
    assert torch.allclose(yarn.freqs[turns < 0.8], base[turns < 0.8] / 4, rtol=1e-14)
    assert bool((yarn.freqs <= base).all()) and bool((yarn.freqs >= base / 4 * (1 - 1e-14)).all())
    assert bool((yarn.freqs[1:] < yarn.freqs[:-1]).all())
    for bad in (dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=130), dict(factor=0.5)):
        with pytest.raises(ValueError):
            api.rope_frequencies(**{"rot_dim": 128, **bad}, device="cpu")


def test_the_rule_of_verification_keeps_the_target_distribution():
    """The reference's walk over every outcome of the drafts and random numbers of a
    small vocabulary: the first new token has the target's probabilities."""
    p, q = torch.tensor([0.5, 0.3, 0.2, 0.0]), torch.tensor([0.2, 0.2, 0.5, 0.1])
    got = torch.zeros(4, dtype=torch.float64)
    steps = 120
    grid = [(i + 0.5) / steps for i in range(steps)]
    target, draft = p.expand(3, 4), q.expand(3, 4)
    for x in range(4):
        for y in range(4):
            weight = float(q[x]) * float(q[y])
            if weight == 0:
                continue
            # both drafts are children of node 0; the three random numbers are independent
            a = 0.0
            take = torch.zeros(4, dtype=torch.float64)
            left = 1.0
            for u, token in ((0, x), (1, y)):
                f = 1.0 if u == 0 else float((p - q).clamp_min(0).sum())
                ok = min(1.0, max(float(p[token]) - a * float(q[token]), 0.0) / (float(q[token]) * f))
                take[token] += left * ok
                left *= 1 - ok
                a += f
            rest = (p.double() - a * q.double()).clamp_min(0)
            got += weight * (take + left * rest / rest.sum())
            # the reference agrees at a few random numbers
            for u in grid[::40]:
                path, token = R.verify(target, draft, [0, x, y], [-1, 0, 0], [0.0, u, u], 0.5, 3)
                first = min(1.0, float(p[x]) / float(q[x]))
                assert (path[:2] == [0, 1]) == (u < first) or abs(u - first) < 1e-6
    assert torch.allclose(got, p.double(), atol=1e-6)


def test_ancestors_and_bits():
    parents = [-1, 0, 0, 1, 2, 9, 5, -3]
    assert R.ancestors(parents, 3) == [3, 1, 0] and R.ancestors(parents, 5) == [5] and R.ancestors(parents, 6) == [6, 5]
    assert R.bits([0, 63, 64], 2) == [(1 | 1 << 63) - (1 << 64), 1] and R.bits([64], 1) == [0]


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(_lib.Rows) == 24 and ctypes.sizeof(_lib.RopeSpec) == 12
    assert ctypes.sizeof(_lib.TreeOpts) == 32 and ctypes.sizeof(_lib.VerifyOpts) == 40
