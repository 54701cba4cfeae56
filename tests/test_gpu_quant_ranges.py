"""Attention over an 8-bit cache at the ends of its numbers (needs a gfx950
GPU): values of V near fp32's largest."""
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
@pytest.mark.parametrize("exponents", [(124, 123), (-3, 124), (126, -20), (0, 1), (-100, -101)])
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
