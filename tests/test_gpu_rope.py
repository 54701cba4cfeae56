"""Rotary positions and the append to the bf16 cache against their definition in
64 bits (needs a gfx950 GPU).

Bounds: the angle's turns are rounded to fp32 (2^-26 of a turn, 2^-23.3 rad), cosine
and sine to a few 2^-24 and once more by the factor, products and sum to 2^-24
each: together within 2^-21 of |x| + |y|, times the factor.  Then one rounding to the
output's type: half its step, and 2^-25 below fp16's normal numbers."""
from __future__ import annotations

import math

import pytest
import torch

import draftref as R
from paper_2606_00024_amd import _lib, api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


def _close(got, ref, size, rounded=True):
    got = got.double().cpu()
    far = size * 2.0 ** -21
    if rounded:
        eps = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}[rounded]
        far = far + eps * (ref.abs() + far) + 2.0 ** -25
    bad = (got - ref).abs() > far
    assert not bool(bad.any()), f"{int(bad.sum())} off, by up to {float(((got - ref).abs() / far).max()):.2f} of the bound"


def _freqs(rot, base=10000.0):
    return api.rope_frequencies(rot, base=base, device=DEV).freqs if rot else torch.empty(0, dtype=torch.float64, device=DEV)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [0, 2, 20, 32, 64, 96, 126, 128])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows(dtype, rot, layout):
    gen = torch.Generator().manual_seed(rot + len(layout))
    for rows, heads in ((1, 1), (7, 5), (130, 12)):
        x = (torch.randn(rows, heads, 128, generator=gen) * 2).to(dtype)
        positions = torch.randint(0, 200000, (rows,), generator=gen).int()
        positions[0] = 2 ** 31 - 1 if rows > 1 else 0
        rope = api.Rope(_freqs(rot), layout, 1.25)
        got = api.rope_rows(x.to(DEV), positions.to(DEV), rope)
        ref, size = R.rotate(x, positions, rope.freqs.cpu(), layout, 1.25)
        assert got.dtype is dtype
        _close(got, ref, size, dtype)


def test_rows_of_one_type_into_another_strided_and_in_place():
    gen = torch.Generator().manual_seed(5)
    rope = api.Rope(_freqs(64), "half", 0.5)
    for a in TYPES:
        for b in TYPES:
            wide = torch.randn(33, 9, 136, generator=gen).to(a).to(DEV)
            x = wide[:, 1:7, :128]
            room = torch.full((33, 8, 144), 7.0, dtype=b, device=DEV)
            out = room[:, 2:8, :128]
            positions = torch.arange(33, dtype=torch.int32, device=DEV) * 1000 - 5000
            assert api.rope_rows(x, positions, rope, out=out) is out
            ref, size = R.rotate(x.cpu(), positions.cpu(), rope.freqs.cpu(), "half", 0.5)
            _close(out, ref, size, b)
            assert bool((room[:, :2] == 7).all()) and bool((room[:, :, 128:] == 7).all())
    for rot, layout in ((128, "half"), (96, "interleaved"), (20, "half"), (20, "interleaved")):
        rope = api.Rope(_freqs(rot), layout)
        x = torch.randn(50, 11, 128, generator=gen).bfloat16().to(DEV)
        positions = torch.randint(0, 5000, (50,), generator=gen).int().to(DEV)
        apart = api.rope_rows(x, positions, rope)
        api.rope_rows(x, positions, rope, out=x)
        assert torch.equal(apart, x)


def test_the_way_back_and_the_gradient():
    gen = torch.Generator().manual_seed(6)
    x = torch.randn(40, 3, 128, generator=gen)
    positions = torch.randint(0, 100000, (40,), generator=gen).int()
    freqs = _freqs(128)
    there = api.rope_rows(x.to(DEV), positions.to(DEV), api.Rope(freqs))
    back = api.rope_rows(there, positions.to(DEV), api.Rope(-freqs)).cpu().double()
    # two rotations, each within 2^-21 of |x| + |y| and a rounding
    assert float((back - x).abs().max()) <= 2 * (2.0 ** -21 + 2.0 ** -24) * 2 * float(x.abs().max()) * math.sqrt(2)
    # the gradient of sum(w . rotated x), against differences of the definition
    w = torch.randn(40, 3, 128, generator=gen)
    grad = api.rope_rows(w.to(DEV), positions.to(DEV), api.Rope(-freqs, "half", 1.5)).cpu().double()
    f = lambda y: (R.rotate(y, positions, freqs.cpu(), "half", 1.5)[0] * w.double()).sum()  # noqa: E731
    for at in ((0, 0, 0), (39, 2, 127), (7, 1, 64)):
        d = torch.zeros(x.shape, dtype=torch.float64)
        d[at] = 0.5     # linear: any step
        assert float(f(x.double() + d) - f(x.double() - d)) == pytest.approx(float(grad[at]), abs=1e-4)


CASES = [  # lens of contexts, nodes, heads (q, kv), page, rows type, rot, layout, by offsets, own positions
    ([0], [1], (4, 1), 16, torch.bfloat16, 128, "half", False, False),
    ([1000], [1], (8, 2), 64, torch.float32, 64, "interleaved", False, False),
    ([5, 0, 31, 700], [3, 3, 3, 3], (6, 2), 16, torch.float16, 96, "half", False, True),
    ([17, 64, 0, 130], [1, 0, 40, 7], (5, 5), 32, torch.bfloat16, 20, "interleaved", True, True),
    ([3, 900], [500, 33], (16, 1), 128, torch.float32, 128, "interleaved", True, False),
    ([10] * 70, [2] * 70, (3, 3), 16, torch.bfloat16, 0, "half", True, False),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("pad", [0, 1])
def test_append(case, pad):
    held, new, (Hq, H), page, dtype, rot, layout, ragged, own_positions = case
    gen = torch.Generator().manual_seed(len(held) * 7 + rot)
    rows = sum(new) + (5 if ragged else 0)
    cpu = R.Cache(gen, [a + b for a, b in zip(held, new)], H, page, pad=pad)
    cache = cpu.to(DEV)
    x = {n: (torch.randn(rows, h, 128, generator=gen) * 2).to(dtype) for n, h in (("q", Hq), ("k", H), ("v", H))}
    first = 2 if ragged else 0
    offsets = torch.tensor([first] + [first + sum(new[: b + 1]) for b in range(len(new))], dtype=torch.int32)
    positions = torch.randint(0, 40000, (rows,), generator=gen).int() if own_positions else None
    rope = api.Rope(_freqs(rot), layout, 0.75) if rot else None
    gpu = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    q_out = torch.full((rows, Hq, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    got = api.rope_append(cache.k, cache.v, gpu(x["k"]), gpu(x["v"]), cache.table, gpu(torch.tensor(held).int()), rope=rope,
                          q=gpu(x["q"]), q_out=q_out, token_offsets=gpu(offsets) if ragged else None,
                          row_positions=gpu(positions))
    assert got is q_out
    k, v, q = cache.k.cpu(), cache.v.cpu(), q_out.cpu()
    touched = torch.zeros(cpu.k.shape[:3], dtype=torch.bool)
    live = torch.zeros(rows, dtype=torch.bool)
    for b, (a, n) in enumerate(zip(held, new)):
        r = torch.arange(n) + int(offsets[b])
        t = torch.arange(a, a + n)
        live[r] = True
        at = positions[r] if own_positions else t
        freqs, scale = (rope.freqs.cpu(), rope.scale) if rope else (torch.empty(0, dtype=torch.float64), 1.0)
        pages, slots = cpu.table[b][t // page].long(), t % page
        touched[pages, :, slots] = True
        for got_rows, source in ((q[r], x["q"]), (k[pages, :, slots], x["k"])):
            ref, size = R.rotate(source[r], at, freqs, layout, scale)
            _close(got_rows, ref, size, torch.bfloat16)
        assert torch.equal(v[pages, :, slots], x["v"][r].to(torch.bfloat16))
    for pool, was in ((k, cpu.k), (v, cpu.v)):
        assert torch.equal(pool[~touched].nan_to_num(123), was[~touched].nan_to_num(123))
    assert bool((q[~live] == 9).all())


def test_append_passes_over_what_does_not_belong():
    """Unused sequences of a padded batch, nodes past the table, bad pages."""
    gen = torch.Generator().manual_seed(3)
    cpu = R.Cache(gen, [16, 16, 16, 16], 2, 16)
    cpu.table[3, 0] = 10 ** 6
    cache = cpu.to(DEV)
    k = torch.randn(8, 2, 128, generator=gen).bfloat16().to(DEV)
    q_out = torch.full((8, 2, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    context = torch.tensor([-1, 15, 3, 3], dtype=torch.int32, device=DEV)
    api.rope_append(cache.k, cache.v, k, k, cache.table, context, q=k, q_out=q_out)
    want_k = cpu.k.clone()
    want_k[cpu.table[2, 0].long(), :, 3:5] = k[4:6].transpose(0, 1).cpu()
    assert torch.equal(cache.k.cpu().nan_to_num(123), want_k.nan_to_num(123))
    assert bool((q_out[:4] == 9).all()) and torch.equal(q_out[4:], k[4:])
    for bad in ([0, 20, 2, 8, 8], [-5, 2, 4, 6, 8], [2 ** 31 - 1, -2 ** 31, 0, 0, 8]):
        offsets = torch.tensor(bad, dtype=torch.int32, device=DEV)   # unspecified, but nothing outside is written
        api.rope_append(cache.k, cache.v, k, k, cache.table, torch.tensor([0, 0, 0, 0], dtype=torch.int32, device=DEV),
                        q=k, q_out=q_out, token_offsets=offsets)
    torch.cuda.synchronize()


def test_append_in_a_graph_and_on_another_stream():
    gen = torch.Generator().manual_seed(4)
    cpu = R.Cache(gen, [40, 40], 2, 16)
    cache = cpu.to(DEV)
    rope = api.rope_frequencies(128)
    x = torch.randn(2, 2, 128, generator=gen).bfloat16().to(DEV)
    context = torch.tensor([7, 20], dtype=torch.int32, device=DEV)
    q_out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        api.rope_append(cache.k, cache.v, x, x, cache.table, context, rope=rope, q=x, q_out=q_out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.rope_append(cache.k, cache.v, x, x, cache.table, context, rope=rope, q=x, q_out=q_out)
    for step in range(3):
        x.copy_(torch.randn(2, 2, 128, generator=gen).bfloat16())
        context += 1
        graph.replay()
        want = api.rope_rows(x, context, rope)
        assert torch.equal(q_out, want)
        for b in range(2):
            t = int(context[b])
            assert torch.equal(cache.k[cache.table[b, t // 16].long(), :, t % 16], want[b])
            assert torch.equal(cache.v[cache.table[b, t // 16].long(), :, t % 16], x[b])
