"""The 8-bit cache at the ends of its numbers (needs a gfx950 GPU): values of V
near fp32's largest, and appends to runs whose scale is no power of two."""
from __future__ import annotations

import sys

import numpy as np
import pytest
import torch

import quantref as R
from paper_2606_00024_amd import _lib, api

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


def _say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def _two_tokens(form, v_low, v_high):
    """Two pages of 64 tokens whose weight lies in one token each: scores of 0
    (V = v_low) and 5 (V = v_high), and of -480 elsewhere.  The second one is
    2^7.2 times the first one's weight."""
    minus = 0xEC if form == "e4m3" else 0xA0    # -96
    one = 0x38 if form == "e4m3" else 1
    k = torch.full((2, 1, 64, 128), minus, dtype=torch.uint8, device=DEV)
    k[0, 0, 7] = 0
    k[1, 0, 50] = one
    v = torch.full((2, 1, 64, 128), one, dtype=torch.uint8, device=DEV)
    ks = torch.ones((2, 1, 1), device=DEV)
    vs = torch.tensor([v_low, v_high], device=DEV).view(2, 1, 1)
    return api.QuantCache(k.view(R.DTYPE[form]), v.view(R.DTYPE[form]), ks, vs)


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("g", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("exponents", [(124, 123), (-3, 124), (126, -20), (80, 79), (79, 85), (0, 1), (-100, -101)])
def test_large_and_small_values(form, g, exponents):
    """600 sequences of two tiles, both of which one wavefront takes without the
    test, so that the first tile's maximum meets the second one's larger score."""
    _say("  values", form, g, exponents)
    low, high = (2.0 ** e for e in exponents)
    cache = _two_tokens(form, low, -1.5 * high)
    B = 600
    q = torch.ones((B, g, 128), dtype=torch.bfloat16, device=DEV)
    table = torch.tensor([[0, 1]], dtype=torch.int32, device=DEV).expand(B, 2).contiguous()
    lens = torch.full((B,), 128, dtype=torch.int32, device=DEV)
    w = np.exp(5.0 - np.logaddexp(0.0, 5.0)), np.exp(-np.logaddexp(0.0, 5.0))
    want = w[0] * -1.5 * high + w[1] * low
    for no_detector in (True, False):
        for order in (0, 1):
            out, lse, _ = api.decode_attention_quant(
                q, cache, table, lens, block_size=64, tau=0.0, phi=0.0, patience=1, dense_order=order,
                softmax_scale=5.0 / 128, no_detector=no_detector)
            got = out.double().cpu().numpy()
            # the score 5 to 2^-24 of itself, three times (scale, product, change of
            # base), moves a weight by 15 * 2^-24 of it; exp2, the parts of P, sums,
            # the join and the division take 16 roundings.  With the test the outputs
            # are a running mean, o + w (o' - o): going forward it holds `low` before
            # the heavier token comes, and rounds its way from there, to 2^-24 of the
            # larger of the two values a step
            size = w[0] * 1.5 * high + w[1] * low if no_detector else max(1.5 * high, low)
            assert np.all(np.abs(got - want) <= 32 * 2.0 ** -24 * size), (got[0, 0, 0], want)
            assert torch.all((lse - float(np.logaddexp(0.0, 5.0))).abs() <= 5 * 16 * 2.0 ** -24)


def _midpoints(form):
    vals = np.unique(R.table(form)[~np.isnan(R.table(form))])
    vals = vals[np.abs(vals) <= R.TOP[form]]
    return np.concatenate([vals, (vals[1:] + vals[:-1]) / 2])


def _host(cache):
    return [t.view(torch.uint8).cpu().numpy().copy() for t in cache[:2]] + [t.cpu().numpy().copy() for t in cache[2:]]


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("run,rows", [(16, 2), (64, 40), (256, 200), (256, 3)])
@pytest.mark.parametrize("wild", [False, True])
def test_append_to_runs_of_any_scale(form, dtype, run, rows, wild):
    """Rows at and next to the midpoints of two codes times the run's scale,
    which is no power of two: the nearest code, ties to even, of the exact
    quotient.  Half of the runs hold the new rows, half grow and round their old
    codes anew."""
    _say("  any scale", form, dtype, run, rows, wild)
    rng = np.random.default_rng(run + rows)
    P = 24
    codes = [rng.integers(0, 256, (P, 1, run, 128), dtype=np.uint8) for _ in range(2)]
    codes = [np.where((c & 127) == 127, 0, c) if form == "e4m3" else np.where(c == 128, 0, c) for c in codes]
    codes = [c.astype(np.uint8) for c in codes]
    # scales of few bits (exact ties) and of 24; those that grow (to 4), such that
    # a code times the scale, over 4, falls next to a midpoint
    scales = rng.uniform(1.0, 2.0, P)
    scales[:8:2] = [1.5, 1.25, 1.0 + 2.0 ** -23, 2.0 - 2.0 ** -23]
    grow = np.arange(P) % 2 == 1
    scales[grow] = (4 * rng.integers(8, 16, grow.sum()) + 2) / rng.choice([72, 80, 88, 96, 104, 112], grow.sum())
    scales = scales.astype(np.float32).reshape(P, 1, 1)
    cache = api.QuantCache(*(torch.from_numpy(c.copy()).to(DEV).view(R.DTYPE[form]) for c in codes),
                           *(torch.from_numpy(scales.copy()).to(DEV) for _ in range(2)))
    host = _host(cache)
    points = _midpoints(form)
    points = points[np.abs(points) < 0.49 * R.TOP[form]]     # (a power of two holds them, at or below the scale)
    x = rng.choice(points, (P, rows, 1, 128)) * scales.reshape(P, 1, 1, 1).astype(np.float64)
    x = x.astype(np.float32)
    step = rng.integers(-1, 2, x.shape)
    x = np.where(step > 0, np.nextafter(x, np.float32(1e9)), np.where(step < 0, np.nextafter(x, np.float32(-1e9)), x))
    x[grow, 0, 0, 0] = 4 * R.TOP[form]
    k = torch.from_numpy(x.reshape(P * rows, 1, 128)).to(DEV).to(dtype)
    if wild:
        k[::3, 0, 5] = float("inf")
        k[1::3, 0, 6] = float("nan")
        k[:, 0, 7] = float("-inf")
    old = run - rows - 3
    positions = np.full(P, old, dtype=np.int32)
    pages = rng.permutation(P).astype(np.int32).reshape(P, 1)
    # rows of sequence b go to page pages[b]: in the order of the pages' scales
    k = k.view(P, rows, 1, 128)[torch.from_numpy(pages[:, 0].astype(np.int64)).to(DEV)].reshape(P * rows, 1, 128).contiguous()
    api.quant_append(cache, k, -k, torch.from_numpy(pages).to(DEV), torch.from_numpy(positions).to(DEV))
    offsets = [b * rows for b in range(P + 1)]
    for i, r in enumerate((k, -k)):
        R.append(host[i], host[2 + i], r.double().cpu().numpy(), pages, positions.tolist(), offsets, form)
    kept = 0
    for got, want in zip(_host(cache), host):
        if want.dtype == np.uint8:
            nan = (form == "e4m3") & ((got & 127) == 127) & ((want & 127) == 127)
            bad = np.argwhere((got != want) & ~nan)
            assert len(bad) == 0, (len(bad), bad[:4].tolist(), [(got[tuple(i)], want[tuple(i)]) for i in bad[:4]])
        else:
            assert np.array_equal(got, want)
            kept += int((want == scales).sum())
    assert kept >= P // 2    # (K and V together)
