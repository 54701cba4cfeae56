"""Writing and reading the 8-bit cache (needs a gfx950 GPU): codes, scales and
rows bit for bit against the definition in 64 bits."""
from __future__ import annotations

import math
import sys

import numpy as np
import pytest
import torch

import quantref as R
from helpers import small_workload
from parity import compare_workload
from paper_2606_00024_amd import _lib, api, workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
ROWS = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


def _i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def _filled(rng, form, P, H, Ps, run):
    """A cache of random codes and power-of-two scales, and its numpy copy."""
    host = []
    for _ in range(2):
        c = rng.integers(0, 256, (P, H, Ps, 128), dtype=np.uint8)
        host.append(np.where((c & 127) == 127, 0, c).astype(np.uint8) if form == "e4m3" else np.where(c == 128, 0, c).astype(np.uint8))
    for _ in range(2):
        host.append(np.exp2(rng.integers(-8, 3, (P, H, Ps // run))).astype(np.float32))
    return _to_gpu(host, form), host


def _to_gpu(host, form):
    return api.QuantCache(*(torch.from_numpy(c.copy()).to(DEV).view(R.DTYPE[form]) for c in host[:2]),
                          *(torch.from_numpy(s.copy()).to(DEV) for s in host[2:]))


def _same(cache, host):
    for name, got, want in zip(cache._fields, cache, host):
        got = (got.view(torch.uint8) if got.dtype != torch.float32 else got).cpu().numpy()
        if want.dtype == np.uint8:
            bad = np.argwhere(got != want)
            # a NaN may carry either sign
            bad = [tuple(i) for i in bad if not (got.dtype == np.uint8 and cache.k.dtype == torch.float8_e4m3fn
                                                and (got[tuple(i)] & 127) == 127 and (want[tuple(i)] & 127) == 127)]
            assert not bad, (name, len(bad), bad[:5], [(got[i], want[i]) for i in bad[:5]])
        else:
            assert np.array_equal(got.view(np.uint32), want.view(np.uint32)), (name, np.argwhere(got != want)[:5])


def _append(cache, host, rows, pages, positions, offsets, form):
    """Both, on rows of a GPU tensor pair."""
    B = pages.shape[0]
    n = rows[0].shape[0]
    api.quant_append(cache, *rows, torch.from_numpy(pages).to(DEV), _i32(positions),
                     token_offsets=_i32(offsets))
    offs = offsets if offsets is not None else [b * (n // B) for b in range(B + 1)]
    pos = positions if positions is not None else [0] * B
    for i in range(2):
        R.append(host[i], host[2 + i], rows[i].double().cpu().numpy(), pages, pos, offs, form)


def _rows(rng, n, H, dtype, size=3.0):
    """Rows of very different sizes, some of them zero."""
    x = rng.standard_normal((n, H, 128)) * np.exp2(rng.integers(-6, 7, (n, H, 1))) * size
    x[rng.random((n, H)) < 0.05] = 0.0
    return torch.from_numpy(x).to(DEV).to(dtype)


def _pages(rng, B, width, spare=1):
    return rng.permutation(B * width + spare)[: B * width].reshape(B, width).astype(np.int32)


CASES = [
    # (Ps, run, positions, counts): one token; one each; long; ragged with empty
    # sequences; starts inside a run, ends inside one, at its ends
    (16, 16, [0], [1]),
    (64, 64, [5, 0, 63, 64, 200], [1, 1, 1, 1, 1]),
    (64, 16, [0, 3, 17], [300, 0, 45]),
    (32, 32, [31, 1, 0, 40], [0, 64, 32, 31]),
    (256, 256, [250, 0], [300, 257]),
    (128, 64, [7, 64, 0, 0], [121, 64, 1, 200]),
    (128, 128, [100], [100]),
    (1024, 256, [1000, 3], [400, 600]),
]


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("dtype", list(ROWS))
@pytest.mark.parametrize("i", range(len(CASES)))
def test_append(form, dtype, i):
    Ps, run, positions, counts = CASES[i]
    _say("  append", form, dtype, CASES[i])
    rng = np.random.default_rng(i)
    B, H = len(counts), 3
    width = -(-max(p + n for p, n in zip(positions, counts)) // Ps) + 1
    cache, host = _filled(rng, form, B * width + 1, H, Ps, run)
    pages = _pages(rng, B, width)
    offsets = np.concatenate([[0], np.cumsum(counts)]).tolist()
    rows = [_rows(rng, offsets[-1], H, ROWS[dtype]) for _ in range(2)]
    _append(cache, host, rows, pages, positions, offsets, form)
    _same(cache, host)      # every byte: slots that get no row keep theirs


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("dtype", list(ROWS))
def test_append_a_prompt_among_decode_steps(form, dtype):
    """Few rows a sequence on average, hundreds of one, some of them not finite."""
    rng = np.random.default_rng(29)
    counts = [1] * 100 + [130] + [2] * 30
    B, H, Ps, run = len(counts), 2, 64, 64
    positions = rng.integers(0, 100, B).tolist()
    cache, host = _filled(rng, form, B * 4 + 1, H, Ps, run)
    pages = _pages(rng, B, 4)
    offsets = np.concatenate([[0], np.cumsum(counts)]).tolist()
    rows = [_rows(rng, offsets[-1], H, ROWS[dtype]) for _ in range(2)]
    for r, (at, bad) in zip(rows, ((3, float("inf")), (150, float("nan")))):
        r[at, 1, 77] = bad
    _append(cache, host, rows, pages, positions, offsets, form)
    _same(cache, host)


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("dtype", list(ROWS))
@pytest.mark.parametrize("run", [128, 256])
def test_append_in_parts_to_long_runs(form, dtype, run):
    """Runs of many rows that come in parts, each larger than the one before,
    some with infinities and NaN; the last row of a run is its largest."""
    rng = np.random.default_rng(run)
    B, H, Ps = 5, 3, 256
    cache, host = _filled(rng, form, B * 6 + 1, H, Ps, run)
    pages = _pages(rng, B, 6)
    positions = [0, 1, 127, 130, 300]
    for step, counts in enumerate([[600, 7, 1, 126, 250], [3, 120, 129, 0, 33], [200, 5, 128, 257, 6]]):
        offsets = np.concatenate([[0], np.cumsum(counts)]).tolist()
        rows = [_rows(rng, offsets[-1], H, ROWS[dtype], 3.0 * 4 ** step) for _ in range(2)]
        rows[0][offsets[1] - 1] *= 16.0
        if step == 1:
            rows[1][offsets[2], 1, 5] = float("-inf")
            rows[1][offsets[3] - 1, 2, 127] = float("nan")
        _append(cache, host, rows, pages, positions, offsets, form)
        _same(cache, host)
        positions = [p + n for p, n in zip(positions, counts)]


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("H", [1, 8])
def test_append_uniform_counts(form, H):
    """No offsets: every sequence has as many rows; no positions: from 0."""
    rng = np.random.default_rng(20)
    cache, host = _filled(rng, form, 4 * 3 + 1, H, 64, 32)
    pages = _pages(rng, 4, 3)
    rows = [_rows(rng, 4 * 70, H, torch.bfloat16) for _ in range(2)]
    _append(cache, host, rows, pages, None, None, form)
    _same(cache, host)


@pytest.mark.parametrize("form", R.FORMATS)
def test_append_token_by_token(form):
    """100 decode steps of 5 sequences, magnitudes that grow and shrink: runs
    grow their scales again and again."""
    rng = np.random.default_rng(21)
    B, H, Ps, run = 5, 2, 64, 32
    cache, host = _filled(rng, form, B * 4 + 1, H, Ps, run)
    pages = _pages(rng, B, 4)
    start = [0, 7, 31, 32, 100]
    for step in range(100):
        rows = [_rows(rng, B, H, torch.bfloat16, size=float(np.exp2(step % 9))) for _ in range(2)]
        _append(cache, host, rows, pages, [s + step for s in start], None, form)
    _same(cache, host)


def test_growing_scales_lose_nothing_in_e4m3():
    """One large token after 15 others moves the scale by 2^9; e4m3 codes of
    values from 2^-2 of the old largest one on stay exact."""
    rng = np.random.default_rng(22)
    cache = api.new_quant_cache(1, 1, 16, device=DEV)
    x = torch.from_numpy(rng.uniform(0.25, 1.0, (15, 1, 128))).to(DEV).bfloat16()
    table = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    api.quant_append(cache, x, x, table, _i32([0]))
    before, _ = api.quant_read(cache, table, _i32([0]), rows=15, dtype=torch.float32)
    api.quant_append(cache, x[:1] * 512, x[:1] * 512, table, _i32([15]))
    after, _ = api.quant_read(cache, table, _i32([0]), rows=15, dtype=torch.float32)
    assert cache.k_scale.item() == 2.0 and torch.equal(before, after)


@pytest.mark.parametrize("form", R.FORMATS)
def test_append_special_values(form):
    """Infinities, NaN, zeros, the smallest and the largest numbers."""
    cache, host = _filled(np.random.default_rng(23), form, 9, 1, 16, 16)
    x = torch.zeros((8 * 4, 1, 128), dtype=torch.float32, device=DEV)
    x[0:4, 0, 0] = math.inf
    x[1, 0, 1] = -math.inf
    x[2, 0, 2] = 3.0
    x[4:8] = math.nan
    x[8, 0, :3] = torch.tensor([math.nan, -5.0, 1e-3], device=DEV)
    x[12, 0, :2] = torch.tensor([3.0e38, -1.0], device=DEV)
    x[16, 0, :2] = torch.tensor([1e-45, 2e-38], device=DEV)
    x[20, 0, :3] = torch.tensor([448.0, -0.0, 447.999], device=DEV)
    x[24, 0, :3] = torch.tensor([127.0, 126.5, -125.5], device=DEV)
    x[28, 0, :3] = torch.tensor([448.5, 2.0 ** -10, 3 * 2.0 ** -11], device=DEV)
    pages = np.arange(8, dtype=np.int32).reshape(8, 1)
    _append(cache, host, [x, -x], pages, None, None, form)
    _same(cache, host)
    # and into runs that hold tokens
    _append(cache, host, [x, -x], pages, [4] * 8, None, form)
    _same(cache, host)


def test_rounding_is_to_nearest_even():
    """Every code and every midpoint between two neighbours, at scale 1."""
    for form in R.FORMATS:
        vals = np.unique(R.table(form)[~np.isnan(R.table(form))])
        vals = vals[np.abs(vals) <= R.TOP[form]]
        points = np.concatenate([vals, (vals[1:] + vals[:-1]) / 2, np.nextafter((vals[1:] + vals[:-1]).astype(np.float32) / 2, np.float32(1e9))])
        x = np.zeros((16 * 128,), dtype=np.float32)
        x[: len(points)] = points
        x[-1] = R.TOP[form]
        rng = np.random.default_rng(0)
        cache, host = _filled(rng, form, 1, 1, 16, 16)
        rows = torch.from_numpy(x.reshape(16, 1, 128)).to(DEV)
        _append(cache, host, [rows, -rows], np.zeros((1, 1), dtype=np.int32), None, None, form)
        assert cache.k_scale.item() == 1.0
        _same(cache, host)


@pytest.mark.parametrize("form", R.FORMATS)
def test_rows_that_are_passed_over(form):
    """Rows before the first and behind the last offset, negative positions,
    tokens past the table's end, page ids out of range: nothing of them is
    written, nothing of them read."""
    rng = np.random.default_rng(24)
    B, H, Ps, run = 6, 2, 32, 16
    cache, host = _filled(rng, form, 20, H, Ps, run)
    pages = rng.permutation(20)[:B * 3].reshape(B, 3).astype(np.int32)
    pages[1, 1], pages[2, 0] = -1, 20          # middle third of b = 1, start of b = 2
    pages[3, 2] = 2 ** 31 - 1
    positions = [0, 10, 5, 80, -1, 90]         # b = 4 unused, b = 5 runs over the table's end
    counts = [33, 60, 40, 16, 7, 50]
    offsets = (np.concatenate([[0], np.cumsum(counts)]) + 3).tolist()
    n = offsets[-1] + 9
    rows = [_rows(rng, n, H, torch.bfloat16) for _ in range(2)]
    _append(cache, host, rows, pages, positions, offsets, form)
    _same(cache, host)
    for dtype in ROWS.values():
        k = torch.full((n, H, 128), 7.0, dtype=dtype, device=DEV)
        v = torch.full_like(k, 7.0)
        api.quant_read(cache, torch.from_numpy(pages).to(DEV), _i32(positions),
                       token_offsets=_i32(offsets), k=k, v=v)
        for got, c, s in ((k, host[0], host[2]), (v, host[1], host[3])):
            want = R.read(c, s, pages, positions, offsets, n, form)
            want = torch.from_numpy(np.where(np.isnan(want), 7.0, want)).to(dtype)
            assert torch.equal(got.cpu(), want)


def test_malformed_offsets_write_nothing_outside():
    """Offsets that decrease, are negative or pass the rows; positions near
    2^31: whatever is written lies in the pools (guard bytes around them stay)."""
    H, Ps = 2, 32
    for offsets, positions in (([5, 3, 40, 10], [0, 0, 0]), ([-4, 100, 7, 2 ** 31 - 1], [2 ** 31 - 1, 1, 2]),
                               ([0, 16, 16, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 20, 60]), ([64, 64, 64, 64], [0, 0, 0])):
        _say("  malformed", offsets, positions)
        buf = torch.full((4, 8 * H * Ps * 128), 0x33, dtype=torch.uint8, device=DEV)
        pools = [buf[i, 2 * H * Ps * 128: 6 * H * Ps * 128].view(4, H, Ps, 128).view(torch.int8) for i in (0, 1)]
        sbuf = torch.full((2, 1000), 5.0, device=DEV)
        scales = [sbuf[i, 100: 100 + 4 * H * 2].view(4, H, 2) for i in (0, 1)]
        cache = api.QuantCache(*pools, *scales)
        table = torch.tensor([[0, 1], [2, 3], [1, 2]], dtype=torch.int32, device=DEV)
        x = torch.ones((64, H, 128), dtype=torch.bfloat16, device=DEV)
        api.quant_append(cache, x, x, table, _i32(positions), token_offsets=_i32(offsets))
        out = torch.full((4, 64, H, 128), 9.0, device=DEV)
        api.quant_read(cache, table, _i32(positions), token_offsets=_i32(offsets), k=out[1], v=out[2])
        torch.cuda.synchronize()
        assert torch.all(buf[:2, : 2 * H * Ps * 128] == 0x33) and torch.all(buf[:2, 6 * H * Ps * 128:] == 0x33)
        assert torch.all(buf[2:] == 0x33) and torch.all(out[0] == 9) and torch.all(out[3] == 9)
        assert torch.all(sbuf[:, :100] == 5) and torch.all(sbuf[:, 100 + 4 * H * 2:] == 5)


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("dtype", list(ROWS))
def test_read(form, dtype):
    """Scales that are no powers of two: one rounding to the rows' type."""
    rng = np.random.default_rng(25)
    B, H, Ps, run = 5, 3, 64, 16
    cache, host = _filled(rng, form, B * 4, H, Ps, run)
    for i in (2, 3):
        host[i][:] = rng.uniform(0.01, 2.0, host[i].shape)
    cache = _to_gpu(host, form)
    pages = _pages(rng, B, 4, spare=0)
    positions, counts = [0, 13, 63, 64, 250], [256, 0, 2, 100, 6]
    offsets = np.concatenate([[0], np.cumsum(counts)]).tolist()
    got = api.quant_read(cache, torch.from_numpy(pages).to(DEV), _i32(positions),
                         token_offsets=_i32(offsets), rows=offsets[-1], dtype=ROWS[dtype])
    for x, c, s in ((got[0], host[0], host[2]), (got[1], host[1], host[3])):
        want = R.read(c, s, pages, positions, offsets, offsets[-1], form)
        # one fp32 product, then one rounding
        want = torch.from_numpy(want.astype(np.float32)).to(ROWS[dtype])
        assert torch.equal(x.cpu(), want)


@pytest.mark.parametrize("form", R.FORMATS)
def test_strides(form):
    """Rows inside a wider projection, pools [page][slot][head][dim], scales of
    another order."""
    rng = np.random.default_rng(26)
    B, H, Ps, run = 3, 2, 32, 32
    cache, host = _filled(rng, form, B * 3, H, Ps, run)
    cache = api.QuantCache(*(t.view(torch.uint8).transpose(1, 2).contiguous().transpose(1, 2).view(t.dtype) for t in cache[:2]),
                           *(t.transpose(0, 1).contiguous().transpose(0, 1) for t in cache[2:]))
    pages = _pages(rng, B, 3, spare=0)
    wide = _rows(rng, 100, 8, torch.bfloat16).view(100, 8 * 128)   # q q q q k k v v
    rows = [wide[:, 512:768].view(100, H, 128), wide[:, 768:].view(100, H, 128)]
    offsets = [0, 60, 60, 100]
    _append(cache, host, rows, pages, [5, 0, 33], offsets, form)
    _same(cache, host)
    out = torch.zeros((100, 8 * 128), dtype=torch.bfloat16, device=DEV)
    api.quant_read(cache, torch.from_numpy(pages).to(DEV), _i32([5, 0, 33]), token_offsets=_i32(offsets),
                   k=out[:, 512:768].view(100, H, 128), v=out[:, 768:].view(100, H, 128))
    for cols, c, s in ((out[:, 512:768], host[0], host[2]), (out[:, 768:], host[1], host[3])):
        want = R.read(c, s, pages, [5, 0, 33], offsets, 100, form)
        assert torch.equal(cols.reshape(100, H, 128).cpu(), torch.from_numpy(want).bfloat16())
    assert not out[:, :512].any()


@pytest.mark.parametrize("B", [64, 65, 300, 5000])
def test_many_sequences(B):
    """More sequences than a wavefront has lanes, most of them empty."""
    rng = np.random.default_rng(27)
    H = 1
    counts = rng.integers(0, 3, B).tolist()
    counts[B // 3: 2 * B // 3] = [0] * (2 * B // 3 - B // 3)
    cache, host = _filled(rng, "e4m3", B + 1, H, 16, 16)
    pages = _pages(rng, B, 1)
    offsets = np.concatenate([[0], np.cumsum(counts)]).tolist()
    positions = rng.integers(0, 13, B).tolist()
    rows = [_rows(rng, offsets[-1], H, torch.bfloat16) for _ in range(2)]
    _append(cache, host, rows, pages, positions, offsets, "e4m3")
    _same(cache, host)
    k, _ = api.quant_read(cache, torch.from_numpy(pages).to(DEV), _i32(positions),
                          token_offsets=_i32(offsets), rows=offsets[-1], dtype=torch.float32)
    want = R.read(host[0], host[2], pages, positions, offsets, offsets[-1], "e4m3")
    assert np.array_equal(k.double().cpu().numpy(), want)


def test_offsets_past_32_bits():
    far = 2_500_000_000 // 16 * 16
    buf = torch.zeros(2 * far + 64 * 128, dtype=torch.uint8, device=DEV)
    pool = buf.as_strided((3, 1, 64, 128), (far, 64 * 128, 128, 1)).view(torch.int8)
    small = api.new_quant_cache(3, 1, 64, dtype=torch.int8, device=DEV)
    rng = np.random.default_rng(28)
    x = _rows(rng, 170, 1, torch.bfloat16)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=DEV)
    api.quant_append(small, x, x, table, None)
    big = small._replace(k=pool, k_scale=torch.zeros_like(small.k_scale))
    api.quant_append(big, x, x, table, None)
    assert torch.equal(big.k, small.k) and torch.equal(big.k_scale, small.k_scale)
    a, _ = api.quant_read(big, table, None, rows=170)
    b, _ = api.quant_read(small, table, None, rows=170)
    assert torch.equal(a, b)


def test_captured_and_replayed():
    """Append and read in a HIP graph: every replay, with new inputs and eager
    work between, gives the eager results."""
    rng = np.random.default_rng(29)
    B, H = 4, 2
    cache = api.new_quant_cache(B * 2, H, 64, device=DEV)
    table = torch.from_numpy(_pages(rng, B, 2, spare=0)).to(DEV)
    positions = _i32([0, 5, 60, 64])
    x = _rows(rng, B, H, torch.bfloat16)
    y = torch.empty((B, H, 128), dtype=torch.float32, device=DEV)
    z = torch.empty_like(y)
    api.quant_append(cache, x, x, table, positions)      # first use outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.quant_append(cache, x, x, table, positions)
        api.quant_read(cache, table, positions, k=y, v=z)
    other = api.new_quant_cache(B * 2, H, 64, device=DEV)
    for t in cache:
        (t.view(torch.uint8) if t.dtype != torch.float32 else t).zero_()
    for step in range(5):
        x.copy_(_rows(rng, B, H, torch.bfloat16))
        positions.add_(1)
        graph.replay()
        api.quant_append(other, x, x, table, positions)
        k, v = api.quant_read(other, table, positions, rows=B, dtype=torch.float32)
        torch.cuda.synchronize()
        assert torch.equal(y, k) and torch.equal(z, v)
        for a, b in zip(cache, other):
            assert torch.equal(a.view(torch.uint8) if a.dtype != torch.float32 else a,
                               b.view(torch.uint8) if b.dtype != torch.float32 else b)


@pytest.mark.parametrize("form,run", [("e4m3", 64), ("int8", 16)])
def test_a_served_batch(form, run):
    """A prompt of every sequence, then decode steps that append and attend, as
    a server uses the three calls: the outputs of every step against the oracle
    on the cache read back."""
    B, H, g, Ps, steps = 3, 2, 4, 64, 6
    rng = np.random.default_rng(30)
    lens = [1000, 1, 130]
    width = 17
    table_np = _pages(rng, B, width)
    table = torch.from_numpy(table_np).to(DEV)
    cache = api.new_quant_cache(B * width + 1, H, Ps, dtype=R.DTYPE[form], scale_tokens=run, device=DEV)
    offsets = np.concatenate([[0], np.cumsum(lens)]).tolist()
    draw = lambda n, h: torch.from_numpy(rng.standard_normal((n, h, 128)).astype(np.float32)).to(DEV).bfloat16()  # noqa: E731
    api.quant_append(cache, draw(offsets[-1], H), draw(offsets[-1], H), table, None,
                     token_offsets=_i32(offsets))
    seq = _i32(lens)
    for step in range(steps):
        api.quant_append(cache, draw(B, H), draw(B, H), table, seq)
        seq = seq + 1
        q = draw(B, H * g)
        got = api.decode_attention_quant(q, cache, table, seq, block_size=64, tau=0.02, phi=0.02, patience=2)
        now = [n + step + 1 for n in lens]
        spans = np.concatenate([[0], np.cumsum(now)]).tolist()
        k, v = api.quant_read(cache, table, None, token_offsets=_i32(spans), rows=spans[-1])
        spec = W.WorkloadSpec(name="served", batch=B, num_q_heads=H * g, num_kv_heads=H,
                              seq_lens=tuple(now), tau=0.02, phi=0.02, patience=2)
        pools = [torch.full((B * width + 1, H, Ps, 128), math.nan, dtype=torch.bfloat16) for _ in range(2)]
        for pool, x in zip(pools, (k.cpu(), v.cpu())):
            for b, n in enumerate(now):
                for t0 in range(0, n, Ps):
                    m = min(Ps, n - t0)
                    pool[table_np[b, t0 // Ps], :, :m] = x[spans[b] + t0: spans[b] + t0 + m].transpose(0, 1)
        wl = W.Workload(spec=spec, q=q.cpu(), k_cache=pools[0], v_cache=pools[1], page_table=table.cpu(),
                        seq_lens=seq.cpu(), block_list=None, block_list_len=None)
        rep = compare_workload(wl, got, tau=0.02, phi=0.02, patience=2, name="quant_served")
        assert rep.ok(), str(rep)
